// Geometry and page layout of the 8-bit paged cache, shared by the kernels that fill, read and manage it.
//
// Pool: codes uint8 [layer][kv head][page][K|V][16 * D], scales float32 [layer][kv head][page][K|V]; a page holds 16 tokens, a
// value is code * scale, codes being int8 (-127..127) or e4m3 bytes. A K block is [token / 8][dim / 16][token % 8][dim % 16], a V
// block [dim][place of the token]: both are rows of 16 bytes in groups of 8 (128 contiguous bytes), which is
//  - what ldmatrix reads without bank conflicts: an 8 x 16-byte matrix of K gives lane (g, t) = (lane / 4, lane % 4) the codes of
//    token g, dims 4t..4t+3 of the chunk, one of V the codes of dim g, places 4t..4t+3;
//  - the tensor cores' core matrix without swizzle (K and V^T both K-major).
// The place of token t in a V row, 4 * ((t % 8) / 2) + 2 * (t / 8) + t % 2, puts the tokens {2t, 2t+1, 2t+8, 2t+9} at 4t..4t+3: those of
// which lane t holds the scores when a 16 x 16 tile of S = Q K^T leaves mma.sync.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "../../include/spec_decode.h"
#include "common.cuh"

namespace spec {

typedef __half f16;
template <> __device__ __forceinline__ float to_f<f16>(f16 v) { return __half2float(v); }
template <> __device__ __forceinline__ f16 from_f<f16>(float v) { return __float2half_rn(v); }

constexpr int CACHE_PAGE = 16;
constexpr float CACHE_FLUSH = 7.888609052210118e-31f;   // 2^-100: a page whose largest magnitude is below is stored as zeros, scale 0
enum { CACHE_INT8 = 0, CACHE_E4M3 = 1 };

__host__ __device__ __forceinline__ int cache_place(int t) { return 4 * ((t & 7) >> 1) + 2 * (t >> 3) + (t & 1); }

struct CacheView {
  uint8_t* codes;
  float* scales;
  int *page_table, *refs, *lens, *status;
  int n_layers, kv, D, n_pages, max_seqs, pages_per_seq;
  // number of the (layer, head, page, K|V) block
  __device__ __host__ __forceinline__ size_t block(int layer, int head, int page, int which) const {
    return ((((size_t)layer * kv + head) * n_pages + page) * 2 + which);
  }
  // sequence number of group b, or -1 (and a mark in the status word)
  __device__ __forceinline__ int sequence(const int* seqs, int b) const {
    const int s = seqs ? seqs[b] : b;
    if (s >= 0 && s < max_seqs) return s;
    set_status(status, ST_BOUNDS, 201, s);
    return -1;
  }
  // page `i` of sequence s, or -1 (and a mark in the status word) where the table holds none
  __device__ __forceinline__ int page(int s, int i) const {
    const int p = i < pages_per_seq ? page_table[(size_t)s * pages_per_seq + i] : -1;
    if (p >= 0 && p < n_pages) return p;
    set_status(status, ST_BOUNDS, 202, i);
    return -1;
  }
  // committed tokens of sequence s, never more than its table can hold
  __device__ __forceinline__ int len(int s) const { return max(0, min(lens[s], pages_per_seq * CACHE_PAGE)); }
};

// Four codes of a word as floats.
template <int FMT> __device__ __forceinline__ void decode4(uint32_t w, float (&f)[4]) {
  if constexpr (FMT == CACHE_INT8) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __uint_as_float(__byte_perm(w ^ 0x80808080u, 0x4b000000u, 0x7440 + i)) - 8388736.f;   // (2^23 + code + 128: the conversion instruction has a quarter of this rate)
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> (16 * i)), __NV_E4M3);
      const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h));
      f[2 * i] = v.x;
      f[2 * i + 1] = v.y;
    }
  }
}
// Four floats in units of the scale as codes: to the nearest, ties to even, held inside the range; NaN becomes code 0 in both formats, so that every stored byte is a finite value.
template <int FMT> __device__ __forceinline__ uint32_t encode4(const float (&f)[4]) {
  uint32_t w = 0;
  if constexpr (FMT == CACHE_INT8) {
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float v = f[i] == f[i] ? fminf(fmaxf(f[i], -127.f), 127.f) : 0.f;
      b[i] = __float_as_uint(v + 12582912.f);                  // (1.5 * 2^23 + v, rounded to even: the low byte is the code)
    }
    w = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
  } else {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float2 v = make_float2(f[2 * i] == f[2 * i] ? f[2 * i] : 0.f, f[2 * i + 1] == f[2 * i + 1] ? f[2 * i + 1] : 0.f);
      w |= (uint32_t)__nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, __NV_E4M3) << (16 * i);
    }
  }
  return w;
}
// The same for finite values times `inv`, none of which passes the range by more than a rounding: one multiply-add a value.
template <int FMT> __device__ __forceinline__ uint32_t encode4_inside(const float (&x)[4], float inv) {
  if constexpr (FMT == CACHE_INT8) {
    uint32_t b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) b[i] = __float_as_uint(fmaf(x[i], inv, 12582912.f));
    return __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
  } else {
    return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(x[0] * inv, x[1] * inv), __NV_SATFINITE, __NV_E4M3) |
           (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(x[2] * inv, x[3] * inv), __NV_SATFINITE, __NV_E4M3) << 16;
  }
}
template <int FMT> __host__ __device__ constexpr float code_max() { return FMT == CACHE_INT8 ? 127.f : 448.f; }

}  // namespace spec
