// Embedding: table rows times a scale, and the table's gradient.
//
// The gradient is the sum of the rows of dX of each word.  The words are sorted
// first (k_embed_sort), so that every row of dE is one sum in registers and one
// store, without atomics, in an order that does not change.  Both kernels are
// bound by memory: the rows once in, the rows of the table once out.
#include <algorithm>

#include "vocab.h"

namespace cavs {
namespace {

// Sizes whose indices the kernels count in 32 bits.  The gradient's sort reads
// every place for each 512 words of the table, once of up to 32 768 places and
// twice of more, which bounds both.
constexpr int kEmbedMax = 1 << 28, kEmbedMaxD = 1 << 14, kGradMax = 1 << 22;
constexpr int kPart = 32;         // rows of a word that one wavefront adds
constexpr int kSortWords = 512;   // most words of a sorting workgroup

// A thread per V elements of X.
template <class E, class X, int V>
__global__ void __launch_bounds__(256) k_embed(int n_words, int D, unsigned total, float scale,
                                               const E* __restrict__ table,
                                               const int* __restrict__ word, X* out, int* err) {
  const unsigned t = blockIdx.x * 256u + threadIdx.x, Q = (unsigned)D / V;
  if (t >= total) return;
  const unsigned i = t / Q, c = (t - i * Q) * V;
  const int w = word[i];
  float v[V];
  if ((unsigned)w < (unsigned)n_words) {
    load_row<V>(table + (size_t)w * D + c, v);
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] *= scale;
  } else {
    if (w != -1) err[1] = 1;
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = 0.f;
  }
  store_row<V>(out + (size_t)i * D + c, v);
}

// Words at i, i + 64, .. (-1 from `to` on), all asked for before the first is
// used: one after the other the sort's second pass took 20 of 26 us of 32 768,
// which are one such load a wavefront.
constexpr int kAhead = 32;
__device__ __forceinline__ void load_words(const int* __restrict__ word, int i, int to, int (&v)[kAhead]) {
#pragma unroll
  for (int k = 0; k < kAhead; ++k) v[k] = i + 64 * k < to ? word[i + 64 * k] : -1;
}

// The places of each word in ascending order: order[start[v] .. start[v + 1]).
// A workgroup takes R adjacent words and reads all n places twice, its sixteen
// wavefronts a contiguous part each: first counting its own words and the places
// of smaller ones (which is where its part of `order` begins), then, with the
// counts scanned over words and wavefronts, giving each place its rank among
// its word's (ballots within the wavefront, whose counts go on in LDS).
__global__ void __launch_bounds__(1024) k_embed_sort(int n, int n_words, int R,
                                                     const int* __restrict__ word, int* start,
                                                     int* order, int* err) {
  __shared__ int cnt[16][kSortWords];
  __shared__ int wsum[16];
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lo = blockIdx.x * R, nr = min(R, n_words - lo);
  const int per = (cdiv_dev(n, 16) + 63) / 64 * 64, from = min(w * per, n), to = min(from + per, n);
  for (int i = lane; i < R; i += 64) cnt[w][i] = 0;   // a wavefront's own counts
  wave_lds_fence();
  int below = 0, v[kAhead];
  bool bad = false;
  for (int i0 = from; i0 < to; i0 += 64 * kAhead) {
    load_words(word, i0 + lane, to, v);
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (i0 + 64 * k >= to) break;
      // what most of the places are is not this workgroup's: a comparison and a
      // count in the scalar unit for each 64 (told apart in lanes, the two passes
      // took 19 us of 32 768 places)
      below += __popcll(__ballot((unsigned)v[k] < (unsigned)lo));
      if (blockIdx.x == 0) bad |= (unsigned)(v[k] + 1) > (unsigned)n_words;
      const unsigned x = (unsigned)v[k] - (unsigned)lo;
      if (__any(x < (unsigned)nr) && x < (unsigned)nr) atomicAdd(&cnt[w][x], 1);
    }
  }
  if (bad) err[1] = 1;
  if (lane == 0) wsum[w] = below;
  __syncthreads();
  int base = 0;
#pragma unroll
  for (int k = 0; k < 16; ++k) base += wsum[k];
  // the words' totals scanned (R is at most 512: a thread each)
  int own = 0;
  if (tid < R)
#pragma unroll
    for (int k = 0; k < 16; ++k) own += cnt[k][tid];
  int incl = own;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(incl, o, kWave);
    if (lane >= o) incl += y;
  }
  __syncthreads();   // wsum has been read
  if (lane == 63) wsum[w] = incl;
  __syncthreads();
  for (int k = 0; k < w; ++k) base += wsum[k];
  if (tid < R) {
    int at = base + incl - own;
    if (tid < nr) start[lo + tid] = at;
    if (tid == nr - 1 && lo + nr == n_words) start[n_words] = at + own;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const int c = cnt[k][tid];
      cnt[k][tid] = at;
      at += c;
    }
  }
  __syncthreads();
  for (int i0 = from; i0 < to; i0 += 64 * kAhead) {
    if (to - from > 64 * kAhead) load_words(word, i0 + lane, to, v);   // else still there
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (i0 + 64 * k >= to) break;
      const unsigned x = (unsigned)v[k] - (unsigned)lo;
      unsigned long long left = __ballot(x < (unsigned)nr), same = 0;
      if (left == 0) continue;
      const bool mine = x < (unsigned)nr;
      while (left) {   // the lanes that share each lane's word
        const int v0 = __builtin_amdgcn_readlane((int)x, __ffsll(left) - 1);
        const unsigned long long m = __ballot(mine && (int)x == v0);
        same = (int)x == v0 ? m : same;
        left &= ~m;
      }
      // the first of them counts them all off and tells them where they begin
      const int rank = __popcll(same & ((1ull << lane) - 1)), first = mine ? __ffsll(same) - 1 : lane;
      int at = 0;
      if (mine && rank == 0) at = atomicAdd(&cnt[w][x], __popcll(same));
      at = __shfl(at, first, kWave);
      if (mine) order[at + rank] = i0 + 64 * k + lane;
    }
  }
}

// The sum of rows order[from .. to) of dX, at most kPart, columns c ..: their
// places in one load, then eight rows in flight, one column block of 64 V to a
// wavefront (20 074 rows of 247 floats: 7 us, 18 with four rows in flight and
// every column to one; 32 768 rows of 2 KB into a table of 100 MB: 41, at 4.1
// TB/s).
template <class X, int V>
__device__ __forceinline__ void add_rows(const X* __restrict__ dX, int D, const int* __restrict__ order,
                                         int from, int to, int c, float (&s)[V]) {
  const int lane = threadIdx.x & 63, n = to - from;
  const int at = lane < n ? order[from + lane] : 0;
#pragma unroll
  for (int k = 0; k < V; ++k) s[k] = 0.f;
  for (int j = 0; j < n; j += 8) {
    // as they are in memory: a conversion here would wait for each in turn
    RawRow<V, X> x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (j + u < n) x[u].load(dX + (size_t)__builtin_amdgcn_readlane(at, j + u) * D + c);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (j + u >= n) break;
      float v[V];
      x[u].floats(v);
#pragma unroll
      for (int k = 0; k < V; ++k) s[k] += v[k];
    }
  }
}

// The first wavefronts take kPart sorted places each: a word that occurs more
// often than kPart times has its share of them summed into part[p][0] (the word
// of the first place) or part[p][1] (one that begins later: at most one such
// word, as it must reach past the end), and begins[p] names the word of that kind
// that begins here, for k_embed_join.  The others take `each` adjacent words and
// write the rows of dE of those that occur at most kPart times (zeros for one
// that does not occur, most of them as a rule).
template <class E, class X, int V>
__global__ void __launch_bounds__(256) k_embed_sum(int n, int n_words, int D, int each, float scale,
                                                   const int* __restrict__ word,
                                                   const int* __restrict__ start,
                                                   const int* __restrict__ order,
                                                   const X* __restrict__ dX, E* dE, float* part,
                                                   int* begins) {
  const int lane = threadIdx.x & 63;
  const int at_ = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  // a row's column blocks are neighbours; past the last column a lane adds its
  // block's first ones and stores nothing
  const int cols = cdiv_dev(D, 64 * V), item = at_ / cols, cb = at_ - item * cols;
  const int c0 = (cb * 64 + lane) * V, c = c0 < D ? c0 : cb * 64 * V;
  float s[V];
  const int parts = cdiv_dev(n, kPart);
  if (item >= parts) {
    const int w0 = (item - parts) * each;   // each is at most 63: a lane for each start
    const int at = start[min(w0 + min(lane, each), n_words)];
    for (int k = 0; k < each && w0 + k < n_words; ++k) {
      const int from = __builtin_amdgcn_readlane(at, k), to = __builtin_amdgcn_readlane(at, k + 1);
      if (to - from > kPart) continue;
      add_rows<X, V>(dX, D, order, from, to, c, s);
#pragma unroll
      for (int i = 0; i < V; ++i) s[i] *= scale;
      if (c0 < D) store_row<V>(dE + (size_t)(w0 + k) * D + c, s);
    }
    return;
  }
  const int p = item, all = start[n_words], lo = p * kPart, hi = min(lo + kPart, all);
  int first = -1;
  if (lo < hi) {
    const int a = __builtin_amdgcn_readfirstlane(word[order[lo]]);
    const int b = __builtin_amdgcn_readfirstlane(word[order[hi - 1]]);
    const int a0 = start[a], a1 = start[a + 1], b0 = start[b], b1 = start[b + 1];
    if (a1 - a0 > kPart) {
      if (a0 == lo) first = a;
      add_rows<X, V>(dX, D, order, lo, min(a1, hi), c, s);
      if (c0 < D) store_row<V>(part + (size_t)p * 2 * D + c, s);
    }
    if (b != a && b1 - b0 > kPart) {
      first = b;
      add_rows<X, V>(dX, D, order, b0, hi, c, s);
      if (c0 < D) store_row<V>(part + (size_t)(p * 2 + 1) * D + c, s);
    }
  }
  if (lane == 0 && cb == 0) begins[p] = first;
}

// dE of the words of more than kPart places: their parts in order, a contiguous
// sixteenth to each wavefront.
template <class E, int V>
__global__ void __launch_bounds__(1024) k_embed_join(int parts, int D, float scale,
                                                     const int* __restrict__ start,
                                                     const int* __restrict__ begins,
                                                     const float* __restrict__ part, E* dE) {
  __shared__ float sums[16][64 * V];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, c = (blockIdx.y * 64 + lane) * V;
  for (int p = blockIdx.x; p < parts; p += gridDim.x) {
    const int v = begins[p];
    if (v < 0) continue;   // the same for the whole workgroup
    const int a = start[v], np = (start[v + 1] - 1) / kPart - p + 1, late = a > p * kPart;
    const int per = cdiv_dev(np, 16), from = min(w * per, np), to = min(from + per, np);
    float s[V] = {};
    if (c < D)
#pragma unroll 4
      for (int q = from; q < to; ++q) {
        float x[V];
        load_row<V>(part + (size_t)(2 * (p + q) + (q == 0 ? late : 0)) * D + c, x);
#pragma unroll
        for (int k = 0; k < V; ++k) s[k] += x[k];
      }
#pragma unroll
    for (int k = 0; k < V; ++k) sums[w][lane * V + k] = s[k];
    __syncthreads();
    if (w == 0 && c < D) {
#pragma unroll
      for (int k = 0; k < V; ++k) {
        s[k] = 0.f;
        for (int i = 0; i < 16; ++i) s[k] += sums[i][lane * V + k];
        s[k] *= scale;
      }
      store_row<V>(dE + (size_t)v * D + c, s);
    }
    __syncthreads();
  }
}

cavs_status embed_args(cavs_ctx* ctx, const cavs_embedding* e, int n) {
  if (!e) return fail(ctx, CAVS_ERR_ARG, "null embedding");
  if ((e->e_type != CAVS_T_F32 && e->e_type != CAVS_T_BF16) ||
      (e->x_type != CAVS_T_F32 && e->x_type != CAVS_T_BF16))
    return fail(ctx, CAVS_ERR_ARG, "unknown element type");
  if (e->n_words <= 0 || e->D <= 0 || n < 0) return fail(ctx, CAVS_ERR_ARG, "bad n_words/D/n");
  if (n > kEmbedMax || e->n_words > kEmbedMax || e->D > kEmbedMaxD)
    return fail(ctx, CAVS_ERR_UNSUPPORTED, "n=%d, n_words=%d, D=%d: at most %d, %d, %d", n, e->n_words,
                e->D, kEmbedMax, kEmbedMax, kEmbedMaxD);
  return CAVS_OK;
}

cavs_status embed_grad_args(cavs_ctx* ctx, const cavs_embedding* e, int n) {
  cavs_status st = embed_args(ctx, e, n);
  if (st != CAVS_OK) return st;
  if (n > kGradMax || e->n_words > kGradMax)
    return fail(ctx, CAVS_ERR_UNSUPPORTED, "gradient of n=%d places, n_words=%d: at most %d each", n,
                e->n_words, kGradMax);
  return CAVS_OK;
}

bool element_aligned(const void* p, int type) {
  return ((uintptr_t)p & (type == CAVS_T_BF16 ? 1 : 3)) == 0;
}

// Elements a thread takes at a time: 16 bytes of the narrower type where rows
// are whole and aligned, else four or one.
int width(int D, const void* a, int ta, const void* b, int tb) {
  const int s = std::max(ta == CAVS_T_BF16 ? 2 : 4, tb == CAVS_T_BF16 ? 2 : 4);
  const bool both = ta == CAVS_T_BF16 && tb == CAVS_T_BF16;
  const uintptr_t at = (uintptr_t)a | (uintptr_t)b;
  if (both && D % 8 == 0 && at % 16 == 0) return 8;
  return D % 4 == 0 && at % (4 * s) == 0 ? 4 : 1;
}

template <class E, class X, int V>
void embed_launch(cavs_ctx* ctx, const cavs_embedding* e, const int* word, int n, void* X_) {
  // 2^31 threads a launch at most
  const int Q = e->D / V, rows = std::max(1, (int)std::min<size_t>((size_t)n, ((size_t)1 << 30) / Q));
  for (int i = 0; i < n; i += rows) {
    const int m = std::min(rows, n - i);
    const unsigned total = (unsigned)m * (unsigned)Q;
    CAVS_LAUNCH("k_embed", (k_embed<E, X, V>), dim3((total + 255) / 256), dim3(256), 0, ctx->stream, e->n_words,
                e->D, total, e->scale, (const E*)e->E, word + i, (X*)X_ + (size_t)i * e->D,
                ctx->dev_err_dev);
  }
}

struct EmbedWs {
  int *start, *order, *begins;
  float* part;
};
size_t embed_ws(const cavs_embedding* e, int n, char* base, EmbedWs& w) {
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t r = o;
    o = align_up(o + bytes, 256);
    return base ? base + r : nullptr;
  };
  const size_t parts = ((size_t)n + kPart - 1) / kPart;
  w.start = (int*)take(((size_t)e->n_words + 1) * 4);
  w.order = (int*)take((size_t)n * 4);
  w.begins = (int*)take(parts * 4);
  w.part = (float*)take(parts * 2 * e->D * 4);
  return o;
}

template <class E, class X, int V>
void embed_grad_launch(cavs_ctx* ctx, const cavs_embedding* e, const int* word, int n, const void* dX,
                       void* dE, const EmbedWs& w) {
  const int parts = cdiv(n, kPart);
  const int cols = cdiv(e->D, 64 * V);
  // some 8192 wavefronts, eight words each at most; more of the largest tables,
  // whose launch stays below 2^32 threads (at most 43, as n_words cols is below 2^30
  // and the parts take 2^25 wavefronts)
  const size_t blocks = (size_t)e->n_words * cols;
  const int each = std::max(std::min(8, std::max(1, (int)(blocks / 8192))), (int)(blocks / (3 << 23) + 1));
  CAVS_LAUNCH("k_embed_sum", (k_embed_sum<E, X, V>), dim3(cdiv(((long)parts + cdiv(e->n_words, each)) * cols, 4)),
              dim3(256), 0, ctx->stream, n, e->n_words, e->D, each, e->scale, word, w.start, w.order,
              (const X*)dX, (E*)dE, w.part, w.begins);
  if (n > kPart)
    CAVS_LAUNCH("k_embed_join", (k_embed_join<E, V>), dim3(std::min(parts, 256), cdiv(e->D, 64 * V)),
                dim3(1024), 0, ctx->stream, parts, e->D, e->scale, w.start, w.begins, w.part, (E*)dE);
}

template <class F>
void by_type(int te, int tx, F f) {
  if (te == CAVS_T_BF16) tx == CAVS_T_BF16 ? f(u16{}, u16{}) : f(u16{}, float{});
  else tx == CAVS_T_BF16 ? f(float{}, u16{}) : f(float{}, float{});
}

}  // namespace

cavs_status embed_run(cavs_ctx* ctx, const cavs_embedding* e, const int* word, int n, void* X) {
  cavs_status st = embed_args(ctx, e, n);
  if (st != CAVS_OK) return st;
  if (n == 0) return CAVS_OK;
  if (!e->E || !word || !X) return fail(ctx, CAVS_ERR_ARG, "E, word and X are required");
  if (!element_aligned(e->E, e->e_type) || !element_aligned(X, e->x_type))
    return fail(ctx, CAVS_ERR_ARG, "E or X is not aligned to its elements");
  const int v = width(e->D, e->E, e->e_type, X, e->x_type);
  by_type(e->e_type, e->x_type, [&](auto te, auto tx) {
    using E = decltype(te);
    using T = decltype(tx);
    if constexpr (sizeof(E) == 2 && sizeof(T) == 2)
      if (v == 8) return embed_launch<E, T, 8>(ctx, e, word, n, X);
    v == 4 ? embed_launch<E, T, 4>(ctx, e, word, n, X) : embed_launch<E, T, 1>(ctx, e, word, n, X);
  });
  CAVS_LAUNCH_CHECK(ctx);
  return CAVS_OK;
}

size_t embed_grad_ws_bytes(const cavs_embedding* e, int n) {
  EmbedWs w;
  return embed_grad_args(nullptr, e, n) == CAVS_OK ? embed_ws(e, n, nullptr, w) : 0;
}

cavs_status embed_grad_run(cavs_ctx* ctx, const cavs_embedding* e, const int* word, int n, const void* dX,
                           void* dE, void* ws, size_t ws_bytes) {
  cavs_status st = embed_grad_args(ctx, e, n);
  if (st != CAVS_OK) return st;
  if (!dE || (n > 0 && (!word || !dX))) return fail(ctx, CAVS_ERR_ARG, "word, dX and dE are required");
  if (!element_aligned(dE, e->e_type) || !element_aligned(dX, e->x_type))
    return fail(ctx, CAVS_ERR_ARG, "dX or dE is not aligned to its elements");
  EmbedWs w;
  const size_t need = embed_ws(e, n, nullptr, w);
  if (!ws || ws_bytes < need)
    return fail(ctx, CAVS_ERR_WORKSPACE, "workspace too small: %zu < %zu", ws_bytes, need);
  if (((uintptr_t)ws & 15) != 0) return fail(ctx, CAVS_ERR_ARG, "ws must be aligned to 16 bytes");
  embed_ws(e, n, (char*)ws, w);
  // about a workgroup per CU, 16 to 512 words each
  const int R = std::min(kSortWords, std::max(16, cdiv(e->n_words, 256)));
  CAVS_LAUNCH("k_embed_sort", k_embed_sort, dim3(cdiv(e->n_words, R)), dim3(1024), 0, ctx->stream, n,
              e->n_words, R, word, w.start, w.order, ctx->dev_err_dev);
  const int v = width(e->D, dE, e->e_type, dX, e->x_type);
  by_type(e->e_type, e->x_type, [&](auto te, auto tx) {
    using E = decltype(te);
    using T = decltype(tx);
    if constexpr (sizeof(E) == 2 && sizeof(T) == 2)
      if (v == 8) return embed_grad_launch<E, T, 8>(ctx, e, word, n, dX, dE, w);
    v == 4 ? embed_grad_launch<E, T, 4>(ctx, e, word, n, dX, dE, w)
           : embed_grad_launch<E, T, 1>(ctx, e, word, n, dX, dE, w);
  });
  CAVS_LAUNCH_CHECK(ctx);
  return CAVS_OK;
}

}  // namespace cavs
