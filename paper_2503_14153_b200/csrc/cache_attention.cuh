// Attention of the rows of a pass over an 8-bit paged cache:
//   o_i = sum_j w_ij v_j / sum_j w_ij,   w_ij = exp(scale * q_i . k_j),
// j over the n cached tokens of the row's sequence (codes * scale of their page and head) and the rows of the pass that the row's mask shows (16-bit, not yet
// in the cache). lse_i = log sum_j w_ij. A row that sees nothing gives zeros and lse -infinity.
#pragma once
#include "cache_common.cuh"
#include "cache_rows.cuh"

namespace spec {

struct CacheAttnArgs {
  CacheView c;
  const void *q, *k, *v;               // [rows][H][D], [rows][kv][D]: strides below, in elements; the last dimension is contiguous
  long long q_row, q_head, k_row, k_head, v_row, v_head;
  void* out;                           // [rows][H][D] contiguous
  float* lse;                          // [rows][H] or nullptr
  const int *seqs, *row_offsets;
  const uint32_t* mask;                // [rows][mask_words] or nullptr (causal)
  int mask_words;
  int rows, batch, H, layer, max_rows;
  float scale;                         // of q . k
};

// sees(i, j): row i of a sequence's rows of the pass sees row j
__device__ __forceinline__ bool row_sees(const uint32_t* mask, int words, int row, int i, int j) {
  if (!mask) return j <= i;
  return (j >> 5) < words && (mask[(size_t)row * words + (j >> 5)] >> (j & 31)) & 1;
}

// ------------------------------------------------------------------ the plain kernel
// A block per (row, head) on CUDA cores, float32 throughout: keys in groups of 128, a thread a key for the scores, a thread one or two dims for the sums.
// It reads the keys once a row, so it is what float32 operands run on (like the float32 kernels of the decode loop), not a path for speed.
constexpr int CAS_THREADS = 128;
template <typename T, int D, int FMT>
__global__ void __launch_bounds__(CAS_THREADS) cache_attention_simple(CacheAttnArgs a) {
  __shared__ float q[D], p[CAS_THREADS], red[8];
  __shared__ float acc_half[D];
  const CacheView& c = a.c;
  const int h = blockIdx.x % a.H, b = blockIdx.z, i = blockIdx.x / a.H + blockIdx.y * (gridDim.x / a.H);
  const int r0 = rows_begin(a.row_offsets, b, a.rows, a.batch), r1 = rows_begin(a.row_offsets, b + 1, a.rows, a.batch);
  const int row = r0 + i, tid = threadIdx.x, kvh = h / (a.H / c.kv);
  if (row >= r1) return;
  const int s = c.sequence(a.seqs, b);
  const int n = s < 0 ? 0 : c.len(s);
  const T* qp = static_cast<const T*>(a.q) + row * a.q_row + h * a.q_head;
  for (int d = tid; d < D; d += CAS_THREADS) q[d] = to_f<T>(qp[d]) * a.scale * 1.44269504088896f;
  float m = -INFINITY, l = 0.f, acc = 0.f;
  constexpr int PARTS = CAS_THREADS / D;          // 2 for D = 64: each half of the threads takes every other key
  const int d = tid % D, part = tid / D;
  for (int k0 = 0; k0 < n + (r1 - r0); k0 += CAS_THREADS) {
    __syncthreads();
    const int j = k0 + tid;
    float z = 0.f;
    bool see = false;
    if (j < n) {
      const int page = c.page(s, j / CACHE_PAGE);
      if (page >= 0) {
        const size_t blk = c.block(a.layer, kvh, page, 0);
        const int t = j % CACHE_PAGE;
        const uint8_t* kp = c.codes + blk * (CACHE_PAGE * D) + (t >> 3) * 8 * D + (t & 7) * 16;
        for (int ch = 0; ch < D / 16; ++ch) {
          const uint4 w = *reinterpret_cast<const uint4*>(kp + ch * 128);
          const uint32_t w4[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            float f[4];
            decode4<FMT>(w4[u], f);
#pragma unroll
            for (int e = 0; e < 4; ++e) z += q[ch * 16 + u * 4 + e] * f[e];
          }
        }
        z *= c.scales[blk];
        see = true;
      }
    } else if (j - n < r1 - r0 && row_sees(a.mask, a.mask_words, row, i, j - n)) {
      const T* kp = static_cast<const T*>(a.k) + (r0 + j - n) * a.k_row + kvh * a.k_head;
      for (int e = 0; e < D; ++e) z += q[e] * to_f<T>(kp[e]);
      see = true;
    }
    float top = see ? z : -INFINITY;
    top = warp_max(top);
    if ((tid & 31) == 0) red[tid >> 5] = top;
    __syncthreads();
    const float mn = fmaxf(fmaxf(m, fmaxf(red[0], red[1])), fmaxf(red[2], red[3]));
    const float ref = mn == -INFINITY ? 0.f : mn;
    const float w = see ? exp2f(z - ref) : 0.f, fix = exp2f(m - ref);
    const float sum = warp_sum(w);
    if ((tid & 31) == 0) red[4 + (tid >> 5)] = sum;
    p[tid] = see ? w : -1.f;
    __syncthreads();
    l = l * fix + ((red[4] + red[5]) + (red[6] + red[7]));
    acc *= fix;
    m = mn;
    const int here = min(CAS_THREADS, n + (r1 - r0) - k0);
    for (int x = part; x < here; x += PARTS) {
      const float pw = p[x];
      if (pw < 0.f) continue;                     // (a masked value may be anything)
      const int key = k0 + x;
      float v;
      if (key < n) {
        const size_t blk = c.block(a.layer, kvh, c.page_table[(size_t)s * c.pages_per_seq + key / CACHE_PAGE], 1);
        const uint8_t code = c.codes[blk * (CACHE_PAGE * D) + d * CACHE_PAGE + cache_place(key % CACHE_PAGE)];
        float f[4];
        decode4<FMT>(code, f);
        v = f[0] * c.scales[blk];
      } else {
        v = to_f<T>(static_cast<const T*>(a.v)[(r0 + key - n) * a.v_row + kvh * a.v_head + d]);
      }
      acc += pw * v;
    }
  }
  if constexpr (PARTS == 2) {
    __syncthreads();
    if (part == 1) acc_half[d] = acc;
    __syncthreads();
    if (part == 1) return;
    acc += acc_half[d];
  }
  const bool none = l == 0.f;
  static_cast<T*>(a.out)[((size_t)row * a.H + h) * D + d] = from_f<T>(none ? 0.f : acc / l);
  if (a.lse && tid == 0) a.lse[(size_t)row * a.H + h] = none ? -INFINITY : (m == -INFINITY ? 0.f : m) * 0.693147180559945f + logf(l);
}

}  // namespace spec
