// Device code shared by the kernels of the 8-bit cache (cache8.hip,
// decode8.hip): lengths, the quantisation of a block, code conversions.
//
// A block is T tokens of one KV head.  With a the largest magnitude of its
// finite elements and top the largest code (127, or e4m3's 448):
//   scale = a / top,  code = rne(x * (top / a)).
// An infinity is taken as +-a, a NaN as 0; a block with a < 2^-100, one without a
// finite element other than 0 among them, gets scale 0 and codes 0 throughout.
// K codes are rows of d bytes; V codes are tiles of 16 tokens, channel by
// channel (byte ((t / 16) * d + c) * 16 + t % 16), so that a lane that wants a
// channel's values for a run of tokens, as P V on the matrix cores does,
// reads them with one 16-byte load.
#pragma once

#include "common.hpp"
#include "internal.hpp"

namespace selkv {

constexpr float kTinyBlock = 0x1p-100f;   // below it top / a nears the end of fp32: the block is stored as zeros

template <int CODE>
__device__ __forceinline__ constexpr float code_top() { return CODE == SELKV_I8 ? 127.f : 448.f; }

// Entries of sequence head / hkv: lens[] where lens is set; negative where that is outside [0, cache_len], the sequence
// then takes no part (appended to at another place it would lose entries).
__device__ __forceinline__ int entries_of(const Lens8& n, uint32_t head, int hkv) {
  if (!n.lens) return n.cache_len;
  const int len = n.lens[head / (uint32_t)hkv];
  return (uint32_t)len <= (uint32_t)n.cache_len ? len : -1;
}

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Four elements of a row in storage type T, raw.  store_streaming: past the caches' replacement order, for rows that
// the call does not read again and that whole wavefronts write line by line.
template <typename T> struct Quad;
template <> struct Quad<float> {
  uint4 w;
  __device__ __forceinline__ void load(const char* p) { w = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void store_streaming(char* p) const {
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4, w), reinterpret_cast<u32x4*>(p));
  }
  __device__ __forceinline__ float get(int e) const {
    return __uint_as_float(e == 0 ? w.x : e == 1 ? w.y : e == 2 ? w.z : w.w);
  }
  // Largest magnitude so far as its bits (they order as the numbers do); bits(m): those of an fp32 number.
  __device__ __forceinline__ uint32_t largest(uint32_t m) const {
    const uint32_t k = 0x7fffffffu;
    return max(max(max(m, w.x & k), max(w.y & k, w.z & k)), w.w & k);
  }
  __device__ static __forceinline__ uint32_t bits(uint32_t m) { return m; }
  __device__ __forceinline__ void set(const float (&x)[4]) {
    w = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};
template <> struct Quad<bf16_t> {
  uint2 w;
  __device__ __forceinline__ void load(const char* p) { w = *reinterpret_cast<const uint2*>(p); }
  __device__ __forceinline__ void store_streaming(char* p) const {
    __builtin_nontemporal_store(__builtin_bit_cast(u32x2, w), reinterpret_cast<u32x2*>(p));
  }
  __device__ __forceinline__ float get(int e) const {
    const uint32_t x = e < 2 ? w.x : w.y;
    return __uint_as_float((e & 1) ? (x & 0xffff0000u) : (x << 16));
  }
  __device__ __forceinline__ uint32_t largest(uint32_t m) const {   // of the even and of the odd elements
    const uint32_t k = 0x7fff7fffu;
    const u16x2 r = __builtin_elementwise_max(__builtin_bit_cast(u16x2, w.x & k), __builtin_bit_cast(u16x2, w.y & k));
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m), r));
  }
  __device__ static __forceinline__ uint32_t bits(uint32_t m) { return max(m << 16, m & 0xffff0000u); }
  __device__ __forceinline__ void set(const float (&x)[4]) {
    w.x = f32_to_bf16(x[0]) | ((uint32_t)f32_to_bf16(x[1]) << 16);
    w.y = f32_to_bf16(x[2]) | ((uint32_t)f32_to_bf16(x[3]) << 16);
  }
};

__device__ __forceinline__ void store16_streaming(char* p, const Chunk16& c) {
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4, c), reinterpret_cast<u32x4*>(p));
}

// |x|, or 0 for an infinity or a NaN.
__device__ __forceinline__ float finite_abs(float x) {
  const float a = fabsf(x);
  return a < __builtin_huge_valf() ? a : 0.f;
}

// Codes of four finite values of a block whose inv is top / a, in the bytes of one word: none is larger than a, so the
// products need no clamp (127 or 448 and an ulp round to the largest code).  int8: adding 1.5 * 2^23 rounds to the
// nearest integer, ties to even, and leaves it in the low byte; the product is rounded on its own, never fused.
template <int CODE>
__device__ __forceinline__ uint32_t encode4(float x0, float x1, float x2, float x3, float inv) {
#pragma clang fp contract(off)
  if constexpr (CODE == SELKV_I8) {
    constexpr float kRound = 12582912.f;
    const uint32_t y0 = __float_as_uint(x0 * inv + kRound), y1 = __float_as_uint(x1 * inv + kRound);
    const uint32_t y2 = __float_as_uint(x2 * inv + kRound), y3 = __float_as_uint(x3 * inv + kRound);
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(y3, y2, 0x0c0c0400u), __builtin_amdgcn_perm(y1, y0, 0x0c0c0400u),
                                 0x05040100u);
  } else {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(x0 * inv, x1 * inv, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(x2 * inv, x3 * inv, w, true);
    return (uint32_t)w;
  }
}

// A value that may be infinite or NaN, brought into [-a, a]: NaN to 0.
__device__ __forceinline__ float tame(float x, float a) { return x == x ? fminf(fmaxf(x, -a), a) : 0.f; }

// The value (without the scale) of byte B of a word of codes.
template <int CODE, int B>
__device__ __forceinline__ float decode1(uint32_t w) {
  if constexpr (CODE == SELKV_I8) return (float)(int8_t)(w >> (8 * B));
  else return __builtin_amdgcn_cvt_f32_fp8((int)w, B);
}

template <int CODE>
__device__ __forceinline__ void decode4(uint32_t w, float (&x)[4]) {
  x[0] = decode1<CODE, 0>(w);
  x[1] = decode1<CODE, 1>(w);
  x[2] = decode1<CODE, 2>(w);
  x[3] = decode1<CODE, 3>(w);
}

// Quantises blocks of K or V by the first 256 threads of a workgroup.  A
// thread holds 16 tokens x 4 channels of its block: d/4 threads side by side
// read a row (256 or 512 bytes together), and each has whole 16-token runs of
// its channels, so V's tiles need no exchange between threads.  Per block
// block/16 * d/4 = 16 .. 256 threads.  Every thread of the workgroup calls it
// (it has barriers); `on`: the thread has a block.
// row(i): address of the thread's channels in token i of its tile; codes (in
// the cache, or LDS to be copied there), scale: of the thread's block.
struct BlockThread {
  int sub, tile, c4;   // block among those of the workgroup, 16-token tile in it, channel / 4
};

template <int D>
__device__ __forceinline__ BlockThread block_thread(int tid, int block) {
  const int per = block / 16 * (D / 4);
  const int u = tid % per;
  return BlockThread{tid / per, u / (D / 4), u % (D / 4)};
}

template <typename T, int D, int CODE, typename Row>
__device__ __forceinline__ void quantise_blocks(bool on, const BlockThread& bt, int block, bool is_v, Row row,
                                                char* codes, float* scale, float (&s_max)[4]) {
  Quad<T> x[16];
  float a = 0.f;
  bool wild = false;   // the thread holds an infinity or a NaN
  if (on) {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i].load(row(i));
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) m = x[i].largest(m);
    a = __uint_as_float(Quad<T>::bits(m));
    wild = Quad<T>::bits(m) >= 0x7f800000u;
    if (wild) {
      a = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) a = fmaxf(a, finite_abs(x[i].get(e)));
    }
  }
  const int per = block / 16 * (D / 4);   // a power of two, 16 .. 256
#pragma unroll
  for (int off = 1; off < 64; off <<= 1)
    if (off < per) a = fmaxf(a, xor_shfl(a, off));
  if (per > 64) {                          // uniform: the waves of a block meet in LDS
    const int wave = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 0 && wave < 4) s_max[wave] = a;
    __syncthreads();
    const int w0 = (wave & 3) & ~(per / 64 - 1);
    for (int w = 0; w < per / 64; ++w) a = fmaxf(a, s_max[w0 + w]);
  }
  if (!on) return;
  const bool tiny = a < kTinyBlock;
  const float inv = tiny ? 0.f : code_top<CODE>() / a;
  if (bt.tile == 0 && bt.c4 == 0) *scale = tiny ? 0.f : a / code_top<CODE>();
  if (wild) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float y[4] = {tame(x[i].get(0), a), tame(x[i].get(1), a), tame(x[i].get(2), a), tame(x[i].get(3), a)};
      x[i].set(y);     // a is an element, so nothing is rounded
    }
  }
  if (!is_v) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      *reinterpret_cast<uint32_t*>(codes + (size_t)(bt.tile * 16 + i) * D + bt.c4 * 4) =
          encode4<CODE>(x[i].get(0), x[i].get(1), x[i].get(2), x[i].get(3), inv);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      Chunk16 ch;
#pragma unroll
      for (int w = 0; w < 4; ++w)
        ch.w[w] = encode4<CODE>(x[4 * w].get(e), x[4 * w + 1].get(e), x[4 * w + 2].get(e), x[4 * w + 3].get(e), inv);
      store16(codes + ((size_t)bt.tile * D + bt.c4 * 4 + e) * 16, ch);
    }
  }
}

}  // namespace selkv
