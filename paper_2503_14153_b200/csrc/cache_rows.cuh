// Rows on their way into the 8-bit paged cache and out of it: rotary positions, quantised store, read-back. All three move
// each value once and are bound by HBM.
#pragma once
#include "cache_common.cuh"

namespace spec {

// ------------------------------------------------------------------ rotary positions
// Pair i of a head, (x1, x2) = (x[i], x[i + rot/2]) in the half layout, (x[2i], x[2i+1]) in the interleaved one, turns by the table's
// angle of the row's position: y1 = x1 c - x2 s, y2 = x2 c + x1 s. Dims from `rot` on, and all of v, are only cast.
constexpr int ROT_THREADS = 128;
constexpr int ROT_HEADS = 4;    // heads whose loads a thread has in flight

struct RotaryArgs {
  const void *q, *k, *v;
  long long q_row, k_row, v_row, q_head, k_head, v_head;   // strides in elements
  void *qo, *ko, *vo;              // contiguous
  const int* positions;
  const float2* table;             // [span][rot / 2] (cos, sin)
  int rows, H, kv, kvv, D, rot, span;    // kvv: heads of v (0: none)
};

template <typename T, int N> struct alignas(sizeof(T) * N) Vec { T x[N]; };

// V pairs a thread: V = 4 where pointers, strides and rot allow 4-element accesses, else 1. A thread keeps its (cos, sin) in registers and
// goes over the heads, ROT_HEADS at a time in flight. blockIdx = (row, part of the heads).
template <typename TI, typename TO, bool IL, int V>
__global__ void __launch_bounds__(ROT_THREADS) rotary_kernel(RotaryArgs a) {
  const int row = blockIdx.x;
  const int pos = a.positions[row];
  const bool inside = pos >= 0 && pos < a.span;     // (a row whose position the table does not hold becomes NaN)
  const int half = a.rot / 2;
  const int per_head = half / V, rest = (a.D - a.rot) / (2 * V), whole = a.D / (2 * V);
  const int heads = a.H + a.kv;
  auto src = [&](int h) -> const TI* {
    return h < a.H ? static_cast<const TI*>(a.q) + row * a.q_row + h * a.q_head : static_cast<const TI*>(a.k) + row * a.k_row + (h - a.H) * a.k_head;
  };
  auto dst = [&](int h) -> TO* {
    return h < a.H ? static_cast<TO*>(a.qo) + ((size_t)row * a.H + h) * a.D : static_cast<TO*>(a.ko) + ((size_t)row * a.kv + h - a.H) * a.D;
  };
  const int lane_heads = ROT_THREADS / per_head > 0 ? ROT_THREADS / per_head : 1;   // heads a sweep of the block covers
  for (int g = threadIdx.x % min(per_head, ROT_THREADS); g < per_head; g += ROT_THREADS) {
    const int hs = threadIdx.x / per_head;
    if (hs >= lane_heads) break;
    float c[V], s[V];
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float2 cs = inside ? a.table[(size_t)pos * half + g * V + j] : make_float2(__int_as_float(0x7fffffff), __int_as_float(0x7fffffff));
      c[j] = cs.x;
      s[j] = cs.y;
    }
    const int step = lane_heads * gridDim.y;
    for (int h0 = blockIdx.y * lane_heads + hs; h0 < heads; h0 += step * ROT_HEADS) {
      Vec<TI, V> lo[ROT_HEADS], hi[ROT_HEADS];
#pragma unroll
      for (int u = 0; u < ROT_HEADS; ++u) {
        const int h = h0 + u * step;
        if (h >= heads) break;
        const TI* p = src(h) + (IL ? 2 * V * g : V * g);
        lo[u] = *reinterpret_cast<const Vec<TI, V>*>(p);
        hi[u] = *reinterpret_cast<const Vec<TI, V>*>(p + (IL ? V : half));
      }
#pragma unroll
      for (int u = 0; u < ROT_HEADS; ++u) {
        const int h = h0 + u * step;
        if (h >= heads) break;
        Vec<TO, V> yl, yh;
        auto el = [&](int i) { return to_f<TI>(i < V ? lo[u].x[i] : hi[u].x[i - V]); };
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const float x1 = IL ? el(2 * j) : el(j), x2 = IL ? el(2 * j + 1) : el(V + j);
          const float y1 = x1 * c[j] - x2 * s[j], y2 = x2 * c[j] + x1 * s[j];
          if constexpr (IL) {
            (2 * j < V ? yl.x[2 * j < V ? 2 * j : 0] : yh.x[2 * j < V ? 0 : 2 * j - V]) = from_f<TO>(y1);
            (2 * j + 1 < V ? yl.x[2 * j + 1 < V ? 2 * j + 1 : 0] : yh.x[2 * j + 1 < V ? 0 : 2 * j + 1 - V]) = from_f<TO>(y2);
          } else {
            yl.x[j] = from_f<TO>(y1);
            yh.x[j] = from_f<TO>(y2);
          }
        }
        TO* o = dst(h) + (IL ? 2 * V * g : V * g);
        *reinterpret_cast<Vec<TO, V>*>(o) = yl;
        *reinterpret_cast<Vec<TO, V>*>(o + (IL ? V : half)) = yh;
      }
    }
  }
  auto copy = [&](const TI* p, TO* o) {
    const Vec<TI, V> x0 = *reinterpret_cast<const Vec<TI, V>*>(p), x1 = *reinterpret_cast<const Vec<TI, V>*>(p + V);
    Vec<TO, V> y0, y1;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      y0.x[j] = from_f<TO>(to_f<TI>(x0.x[j]));
      y1.x[j] = from_f<TO>(to_f<TI>(x1.x[j]));
    }
    *reinterpret_cast<Vec<TO, V>*>(o) = y0;
    *reinterpret_cast<Vec<TO, V>*>(o + V) = y1;
  };
  const int at = blockIdx.y * ROT_THREADS + threadIdx.x, all = gridDim.y * ROT_THREADS;
#pragma unroll 2
  for (int i = at; i < a.kvv * whole; i += all) {
    const int h = i / whole, d = (i - h * whole) * 2 * V;
    copy(static_cast<const TI*>(a.v) + row * a.v_row + h * a.v_head + d, static_cast<TO*>(a.vo) + ((size_t)row * a.kvv + h) * a.D + d);
  }
  for (int i = at; i < heads * rest; i += all) {
    const int h = i / rest, d = a.rot + (i - h * rest) * 2 * V;
    copy(src(h) + d, dst(h) + d);
  }
}

// (cos, sin) of every position below `span` and pair: the angle position * freq[i] and the functions in double, times `gain`, rounded once.
__global__ void rotary_table_kernel(float2* table, const double* __restrict__ freq, int span, int half, double gain) {
  const long long n = (long long)span * half;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long long)gridDim.x * blockDim.x) {
    double s, c;
    sincos((double)(i / half) * freq[i % half], &s, &c);
    table[i] = make_float2((float)(c * gain), (float)(s * gain));
  }
}

// ------------------------------------------------------------------ store
// Rows path[b][0..count) of sequence b's rows of the pass (rows 0..count without a path) become tokens len - count .. len - 1. A warp owns the
// K or the V block of one (layer, head, page): 16 rows in registers, the scale from their largest magnitude by a warp reduction, one write. A page
// that held tokens before (the first one, where the sequence does not end at a page's end) keeps a scale at least as large, and its older codes are
// rounded once more where the scale grew. Rows after the sequence's end are written as zeros.
struct StoreArgs {
  CacheView c;
  const void *k, *v;                   // [layers][rows][kv][D]
  long long k_layer, k_row, k_head, v_layer, v_row, v_head;
  const int *seqs, *row_offsets, *counts, *path;
  int rows, batch, layer0, path_len, slots;   // slots: pages a sequence's rows may touch
};

__device__ __forceinline__ int rows_begin(const int* row_offsets, int b, int rows, int batch) {
  if (!row_offsets) return b * (rows / batch);
  return b >= batch ? min(rows, max(0, row_offsets[batch])) : min(rows, max(0, row_offsets[b]));
}

constexpr int STORE_WARPS = 4;

// D / 32 16-byte chunks a lane and block (a block has 16 rows x D/16 chunks)
template <typename T, int D, int FMT>
__global__ void __launch_bounds__(32 * STORE_WARPS) cache_store_kernel(StoreArgs a) {
  constexpr int CH = D / 32;
  const CacheView& c = a.c;
  const int b = blockIdx.x / a.slots, slot = blockIdx.x % a.slots, lane = threadIdx.x & 31;
  const int unit = blockIdx.y * STORE_WARPS + (threadIdx.x >> 5);
  if (unit >= 2 * c.kv) return;
  const int head = unit >> 1, which = unit & 1, layer = blockIdx.z;
  const int s = c.sequence(a.seqs, b);
  if (s < 0) return;
  const int len = c.len(s), count = max(0, min(a.counts[b], len)), first = len - count;
  const int p = first / CACHE_PAGE + slot;
  if (count == 0 || p * CACHE_PAGE >= len) return;
  const int page = c.page(s, p);
  if (page < 0) return;
  const int base = p * CACHE_PAGE;     // token of the page's first row
  const int r0 = rows_begin(a.row_offsets, b, a.rows, a.batch), r1 = rows_begin(a.row_offsets, b + 1, a.rows, a.batch);
  // the row of the pass that becomes row t of the page: -1 not a new one
  int mine = -1;
  if (lane < CACHE_PAGE && base + lane >= first && base + lane < len) {
    const int i = base + lane - first;
    const int r = r0 + (a.path ? (i < a.path_len ? a.path[(size_t)b * a.path_len + i] : -1) : i);
    if (r >= r0 && r < r1) mine = r;
    else set_status(c.status, ST_BOUNDS, 203, i);
  }
  const size_t blk = c.block(a.layer0 + layer, head, page, which);
  uint4* code = reinterpret_cast<uint4*>(c.codes + blk * (CACHE_PAGE * D));
  const bool held = base < first;
  const float was = held ? c.scales[blk] : 0.f;
  float x[CH][16];                     // chunk i of the lane: number lane + 32 i (K) or the dims 2 lane + 64 (i / 2) + i % 2 (V)
  float top = 0.f;
  const T* in = static_cast<const T*>(which ? a.v : a.k) + layer * (which ? a.v_layer : a.k_layer) + head * (which ? a.v_head : a.k_head);
  const long long rs = which ? a.v_row : a.k_row;
  auto chunk_number = [&](int i) { return which ? 2 * lane + 64 * (i >> 1) + (i & 1) : lane + 32 * i; };
  if (which == 0) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int j = lane + 32 * i, t = (j / (D / 2)) * 8 + (j & 7), d = ((j >> 3) % (D / 16)) * 16;
      const int r = __shfl_sync(0xffffffffu, mine, t);
      if (r >= 0) {
        constexpr int N = 16 / sizeof(T);
#pragma unroll
        for (int u = 0; u < 16 / N; ++u) {
          const Vec<T, N> w = *reinterpret_cast<const Vec<T, N>*>(in + r * rs + d + u * N);
#pragma unroll
          for (int e = 0; e < N; ++e) x[i][u * N + e] = to_f<T>(w.x[e]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) x[i][e] = 0.f;
      }
    }
  } else {
#pragma unroll
    for (int t = 0; t < CACHE_PAGE; ++t) {
      const int r = __shfl_sync(0xffffffffu, mine, t);
#pragma unroll
      for (int i = 0; i < CH; i += 2) {
        Vec<T, 2> w{};
        if (r >= 0) w = *reinterpret_cast<const Vec<T, 2>*>(in + r * rs + 2 * lane + 32 * i);
        x[i][cache_place(t)] = r >= 0 ? to_f<T>(w.x[0]) : 0.f;
        x[i + 1][cache_place(t)] = r >= 0 ? to_f<T>(w.x[1]) : 0.f;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < CH; ++i)
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float m = fabsf(x[i][e]);
      top = m < INFINITY ? fmaxf(top, m) : top;          // (neither infinities nor NaN count for the scale)
    }
  top = warp_max(top);
  const float now = fmaxf(was, top < CACHE_FLUSH ? 0.f : top / code_max<FMT>());
  const float inv = now > 0.f ? 1.f / now : 0.f, again = now > 0.f ? was / now : 0.f;
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int j = chunk_number(i);
    uint4 old = make_uint4(0, 0, 0, 0);
    if (held) old = code[j];
    uint32_t w[4];
    const uint32_t o4[4] = {old.x, old.y, old.z, old.w};
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      float f[4], g[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) f[e] = x[i][4 * u + e] * inv;
      if (held) {
        decode4<FMT>(o4[u], g);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          // token of this value: of the chunk (K), or by its place (V: the inverse of cache_place)
          const int pl = 4 * u + e;
          const int t = which ? 2 * (pl >> 2) + 8 * ((pl >> 1) & 1) + (pl & 1) : (j / (D / 2)) * 8 + (j & 7);
          if (base + t < first) f[e] = g[e] * again;
        }
      }
      w[u] = encode4<FMT>(f);
    }
    code[j] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  if (lane == 0) c.scales[blk] = now;
}

// ------------------------------------------------------------------ read
// Tokens start[b] .. start[b] + window - 1 of every sequence and layer, decoded; tokens past the sequence's end are zeros. A warp decodes one block.
struct ReadArgs {
  CacheView c;
  void *k, *v;                         // [layers][batch][window][kv][D]
  const int *seqs, *start;
  int batch, window, layer0, slots;
};

template <typename T, int D, int FMT>
__global__ void __launch_bounds__(32 * STORE_WARPS) cache_read_kernel(ReadArgs a) {
  constexpr int CH = D / 32;
  const CacheView& c = a.c;
  const int b = blockIdx.x / a.slots, slot = blockIdx.x % a.slots, lane = threadIdx.x & 31;
  const int unit = blockIdx.y * STORE_WARPS + (threadIdx.x >> 5);
  if (unit >= 2 * c.kv) return;
  const int head = unit >> 1, which = unit & 1, layer = blockIdx.z;
  const int start = a.start ? max(0, a.start[b]) : 0;
  const int p = start / CACHE_PAGE + slot, base = p * CACHE_PAGE;
  if (base >= start + a.window) return;
  const int s = c.sequence(a.seqs, b);
  const int len = s < 0 ? 0 : c.len(s);
  const int page = base < len ? c.page(s, p) : -1;
  T* out = static_cast<T*>(which ? a.v : a.k) + (((size_t)layer * a.batch + b) * a.window * c.kv + head) * D;
  const size_t blk = page < 0 ? 0 : c.block(a.layer0 + layer, head, page, which);
  const uint4* code = reinterpret_cast<const uint4*>(c.codes + blk * (CACHE_PAGE * D));
  const float scale = page < 0 ? 0.f : c.scales[blk];
  float x[CH][16];
#pragma unroll
  for (int i = 0; i < CH; ++i) {
    const int j = which ? 2 * lane + 64 * (i >> 1) + (i & 1) : lane + 32 * i;
    uint4 w = make_uint4(0, 0, 0, 0);
    if (page >= 0) w = code[j];
    const uint32_t w4[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      float g[4];
      decode4<FMT>(w4[u], g);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[i][4 * u + e] = g[e] * scale;
    }
  }
  auto row_of = [&](int t) -> T* {
    const int i = base + t - start;
    return i >= 0 && i < a.window ? out + (size_t)i * c.kv * D : nullptr;
  };
  if (which == 0) {
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      const int j = lane + 32 * i, t = (j / (D / 2)) * 8 + (j & 7), d = ((j >> 3) % (D / 16)) * 16;
      T* o = row_of(t);
      if (!o) continue;
      constexpr int N = 16 / sizeof(T);
#pragma unroll
      for (int u = 0; u < 16 / N; ++u) {
        Vec<T, N> w;
#pragma unroll
        for (int e = 0; e < N; ++e) w.x[e] = from_f<T>(base + t < len ? x[i][u * N + e] : 0.f);
        *reinterpret_cast<Vec<T, N>*>(o + d + u * N) = w;
      }
    }
  } else {
#pragma unroll
    for (int t = 0; t < CACHE_PAGE; ++t) {
      T* o = row_of(t);
      if (!o) continue;
#pragma unroll
      for (int i = 0; i < CH; i += 2) {
        Vec<T, 2> w;
        w.x[0] = from_f<T>(base + t < len ? x[i][cache_place(t)] : 0.f);
        w.x[1] = from_f<T>(base + t < len ? x[i + 1][cache_place(t)] : 0.f);
        *reinterpret_cast<Vec<T, 2>*>(o + 2 * lane + 32 * i) = w;
      }
    }
  }
}

}  // namespace spec
