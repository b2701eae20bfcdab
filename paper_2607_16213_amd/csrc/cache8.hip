// selkv_cache8_write and selkv_cache8_read: rows of a KV cache to 8-bit codes
// with one scale per block of tokens and KV head, and back.
//
// Write: a workgroup of 256 threads takes whole blocks (1 .. 16 of them, by
// their size).  A block is read once, its rows stay in registers while the
// largest magnitude is found, and its codes meet in LDS in the order of the
// cache, to be stored line by line: d * sizeof(T) bytes read and d written per
// row, with no scratch and one launch for K and V.
// The rows of the first block may lie in the tail (the open block of earlier
// calls); the workgroup that reads them there is the one that later overwrites
// the tail with the call's own incomplete block, behind a barrier.
// Read: a thread takes 16 tokens x 4 channels, as the write does.
// Both are bound by the memory they move.  Stores pass the caches' replacement
// order by (nothing here is read again): 32 layers x 8 heads x 25600 rows of
// bf16 are written in 890 us, 5.7 TB/s, against 914 with ordinary stores (and
// 4% more where each thread stores its codes as it holds them, 16-byte pieces
// 64 bytes apart); a layer of them is read back in 24.9 us, 6.3 TB/s, against
// 33.9.  A finite block's codes need no clamp and few instructions a value
// (cache8.hpp), which short calls feel: 8191 rows of a layer take 10.1 us, 11.4
// with clamps and conversions one by one.
#include <float.h>

#include "cache8.hpp"

namespace selkv {
namespace {

constexpr int kThreads = 256;

struct WriteArgs {
  Cache8 c;
  Lens8 n;
  const int32_t* counts;
  const char* K_new;
  const char* V_new;
  int n_new, hkv;
};

template <typename T, int D, int CODE>
__global__ __launch_bounds__(kThreads) void cache8_write_kernel(WriteArgs a) {
  constexpr int RB = D * (int)sizeof(T);
  __shared__ float s_max[4];
  __shared__ __align__(16) char s_codes[kThreads * 64];   // the workgroup's codes, as they lie in the cache
  const bool is_v = blockIdx.z != 0;
  const uint32_t head = blockIdx.y;
  const int block = a.c.block, cap = a.c.capacity;
  const int len = entries_of(a.n, head, a.hkv);
  if (len < 0) return;
  int cnt = a.n_new;
  if (a.counts) cnt = max(0, min(a.counts[head / (uint32_t)a.hkv], cnt));
  cnt = min(cnt, cap - len);
  const int r0 = len % block, fb = len / block;   // rows in the tail, first block the call may complete
  const int full = (len + cnt) / block - fb;      // blocks that it completes
  const int per_wg = kThreads / (block / 16 * (D / 4));
  if (blockIdx.x > 0 && (int64_t)blockIdx.x * per_wg >= full) return;

  char* tail = (is_v ? a.c.v_tail : a.c.k_tail) + (size_t)head * block * RB;
  const char* fresh = (is_v ? a.V_new : a.K_new) + (size_t)head * a.n_new * RB;
  if (full > 0) {
    const BlockThread bt = block_thread<D>(threadIdx.x, block);
    const int i_blk = blockIdx.x * per_wg + bt.sub;
    const int rel0 = i_blk * block + bt.tile * 16;   // the thread's first token, counted from block fb's first
    const int byte = bt.c4 * 4 * (int)sizeof(T);
    quantise_blocks<T, D, CODE>(
        i_blk < full, bt, block, is_v,
        [&](int i) {
          const int rel = rel0 + i;
          return (rel < r0 ? tail + (size_t)rel * RB : fresh + (size_t)(rel - r0) * RB) + byte;
        },
        s_codes + (size_t)bt.sub * block * D, (is_v ? a.c.v_scale : a.c.k_scale) + (size_t)head * (cap / block) + fb + i_blk,
        s_max);
    __syncthreads();
    const int first = blockIdx.x * per_wg;
    char* to = (is_v ? a.c.V : a.c.K) + ((size_t)head * cap + (size_t)(fb + first) * block) * D;
    const int bytes = min(per_wg, full - first) * block * D;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int at = (s * kThreads + (int)threadIdx.x) * 16;
      if (at < bytes) store16_streaming(to + at, load16(s_codes + at));
    }
  }
  if (blockIdx.x > 0) return;
  // the rows of the last, incomplete block: behind those that the tail holds, or from its start
  __syncthreads();
  const int at = full > 0 ? 0 : r0;
  const int from = full > 0 ? full * block - r0 : 0;
  const int rows = full > 0 ? (len + cnt) % block : cnt;
  for (int i = threadIdx.x; i < rows * (RB / 16); i += kThreads)
    store16(tail + (size_t)at * RB + (size_t)i * 16, load16(fresh + (size_t)from * RB + (size_t)i * 16));
}

struct ReadArgs {
  Cache8 c;
  Lens8 n;
  char* K_out;
  char* V_out;
  int first, count, hkv;
};

template <typename T, int D, int CODE>
__global__ __launch_bounds__(kThreads) void cache8_read_kernel(ReadArgs a) {
  constexpr int RB = D * (int)sizeof(T);
  constexpr int kTiles = kThreads / (D / 4);   // 16-token tiles of a workgroup
  const bool is_v = blockIdx.z != 0;
  const uint32_t head = blockIdx.y;
  const int len = entries_of(a.n, head, a.hkv);
  const int block = a.c.block, cap = a.c.capacity;
  const int end = min(a.first + a.count, len);
  const int c4 = threadIdx.x % (D / 4);
  const int t0 = (a.first / 16 + blockIdx.x * kTiles + threadIdx.x / (D / 4)) * 16;
  if (t0 >= end) return;
  const int whole = len / block * block;       // entries held as codes, a multiple of 16: a tile is one or the other
  char* out = (is_v ? a.V_out : a.K_out) + (size_t)head * a.count * RB + c4 * 4 * sizeof(T);
  Quad<T> x[16];
  if (t0 < whole) {
    const float sc = (is_v ? a.c.v_scale : a.c.k_scale)[(size_t)head * (cap / block) + t0 / block];
    const char* codes = (is_v ? a.c.V : a.c.K) + ((size_t)head * cap + t0) * D;
    float f[16][4];
    if (!is_v) {
      uint32_t w[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) w[i] = *reinterpret_cast<const uint32_t*>(codes + (size_t)i * D + c4 * 4);
#pragma unroll
      for (int i = 0; i < 16; ++i) decode4<CODE>(w[i], f[i]);
    } else {
      Chunk16 ch[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) ch[e] = load16(codes + (c4 * 4 + e) * 16);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          float y[4];
          decode4<CODE>(ch[e].w[w], y);
#pragma unroll
          for (int i = 0; i < 4; ++i) f[4 * w + i][e] = y[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[i][e] *= sc;
        // 127 * (a / 127) may round past the largest number where a is next to it
        if constexpr (sizeof(T) == 4) f[i][e] = fminf(fmaxf(f[i][e], -FLT_MAX), FLT_MAX);
      }
      x[i].set(f[i]);
    }
  } else {
    const char* tail = (is_v ? a.c.v_tail : a.c.k_tail) + ((size_t)head * block + (t0 - whole)) * RB + c4 * 4 * sizeof(T);
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i].load(tail + (size_t)min(i, end - 1 - t0) * RB);
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int e = t0 + i;
    if (e >= a.first && e < end) x[i].store_streaming(out + (size_t)(e - a.first) * RB);
  }
}

template <typename T, int D>
void write_td(const dim3& grid, const WriteArgs& a, hipStream_t st) {
  if (a.c.code == SELKV_I8) hipLaunchKernelGGL((cache8_write_kernel<T, D, SELKV_I8>), grid, dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL((cache8_write_kernel<T, D, SELKV_E4M3>), grid, dim3(kThreads), 0, st, a);
}

template <typename T, int D>
void read_td(const dim3& grid, const ReadArgs& a, hipStream_t st) {
  if (a.c.code == SELKV_I8) hipLaunchKernelGGL((cache8_read_kernel<T, D, SELKV_I8>), grid, dim3(kThreads), 0, st, a);
  else hipLaunchKernelGGL((cache8_read_kernel<T, D, SELKV_E4M3>), grid, dim3(kThreads), 0, st, a);
}

}  // namespace

hipError_t launch_cache8_write(int64_t heads, int hkv, int d, int dtype, const Cache8& c, const Lens8& n,
                               const int32_t* counts, const void* K_new, const void* V_new, int n_new,
                               hipStream_t st) {
  const WriteArgs a{c, n, counts, static_cast<const char*>(K_new), static_cast<const char*>(V_new), n_new, hkv};
  // blocks that a sequence may complete: known, or at most those of a tail that lacks one row
  const int open = n.lens ? c.block - 1 : n.cache_len % c.block;
  const int64_t full = ((int64_t)open + n_new) / c.block;
  const int per_wg = kThreads / (c.block / 16 * (d / 4));
  const dim3 grid((unsigned)(full > 0 ? (full + per_wg - 1) / per_wg : 1), (unsigned)heads, 2);
  if (dtype == SELKV_BF16) {
    if (d == 128) write_td<bf16_t, 128>(grid, a, st);
    else write_td<bf16_t, 64>(grid, a, st);
  } else {
    if (d == 128) write_td<float, 128>(grid, a, st);
    else write_td<float, 64>(grid, a, st);
  }
  return hipGetLastError();
}

hipError_t launch_cache8_read(int64_t heads, int hkv, int d, int dtype, const Cache8& c, const Lens8& n, void* K_out,
                              void* V_out, int first, int count, hipStream_t st) {
  const ReadArgs a{c, n, static_cast<char*>(K_out), static_cast<char*>(V_out), first, count, hkv};
  const int tiles = (first + count + 15) / 16 - first / 16, per_wg = kThreads / (d / 4);
  const dim3 grid((unsigned)((tiles + per_wg - 1) / per_wg), (unsigned)heads, 2);
  if (dtype == SELKV_BF16) {
    if (d == 128) read_td<bf16_t, 128>(grid, a, st);
    else read_td<bf16_t, 64>(grid, a, st);
  } else {
    if (d == 128) read_td<float, 128>(grid, a, st);
    else read_td<float, 64>(grid, a, st);
  }
  return hipGetLastError();
}

}  // namespace selkv
