// The norm of all gradients together, and the gradients scaled so that it stays
// below a limit:
//
//   norm = |scale| sqrt(sum g^2),   out = g scale min(1, max_norm / norm)
//
// Squares and their sums are kept in 64 bits, which no gradient overflows; every
// sum has one order, whatever runs when.  Bound by memory: the gradients are read
// once for the sum and once more to be scaled.
#include <algorithm>
#include <cmath>
#include <iterator>

#include "vocab.h"

namespace cavs {
namespace {

constexpr int kSlots = 1024;     // workgroups of a launch, each with a partial sum
constexpr int kThreads = 512;
constexpr int kChunk = kThreads * 8;   // elements that a workgroup takes at a time
constexpr int kSet = 160;        // gradients whose list is an argument of a launch
constexpr int kTable = 4096;     // gradients of a table in the workspace
// Elements that a launch writes from which on they go past the caches: fewer fit into
// them beside what the next step reads (norm and scaling together, stores into the
// caches and past them: 12 million in fp32 31.3 us and 26.9, 111 million in bf16 132
// and 108).  Elements, not chunks: a tensor of any size has one at least.
constexpr long long kFar = 8 << 20;

// Gradients of a launch; end[k]: chunks up to and with the k-th's.
struct ClipSet {
  const void* g[kSet];
  void* out[kSet];
  uint32_t n[kSet];    // 0: 2^32
  uint32_t end[kSet];
  uint32_t gbf[kSet / 32], obf[kSet / 32];
  int count;
};
static_assert(sizeof(ClipSet) <= 3968, "kernel arguments");

// The same in the workspace, of all gradients, which the norm's launches leave for the
// one that scales.
struct ClipEntry {
  const void* g;
  void* out;
  long long n;
  uint32_t end, types;   // bit 0: g is bf16, 1: out is
};

__device__ __forceinline__ long long clip_size(uint32_t n) { return n ? n : 1ll << 32; }

// Vectors at any address that is aligned to its elements.
template <class T, int V>
struct Vec {
  typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};

// Eight adjacent elements as they are in memory.
template <class T>
struct Vec8 {
  typedef typename Vec<T, 16 / sizeof(T)>::type part;
  part x[sizeof(T) / 2];
  __device__ __forceinline__ void load(const T* p) {
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) x[i] = reinterpret_cast<const part*>(p)[i];
  }
  __device__ __forceinline__ void floats(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if constexpr (sizeof(T) == 4) v[i] = x[i / 4][i % 4];
      else v[i] = __uint_as_float((uint32_t)x[0][i] << 16);
    }
  }
};
__device__ __forceinline__ float one_float(float v) { return v; }
__device__ __forceinline__ float one_float(u16 v) { return __uint_as_float((uint32_t)v << 16); }

// FAR: past the caches, which then keep what is read next (the gradients themselves,
// for the pass that scales them); from kFar on, where the figures are.
template <bool FAR, class V>
__device__ __forceinline__ void put(V* p, V v) {
  if constexpr (FAR) __builtin_nontemporal_store(v, p);
  else *p = v;
}
template <bool FAR, class T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
    typedef typename Vec<float, 4>::type f4;
    put<FAR>(reinterpret_cast<f4*>(p), f4{v[0], v[1], v[2], v[3]});
    put<FAR>(reinterpret_cast<f4*>(p + 4), f4{v[4], v[5], v[6], v[7]});
  } else {
    typedef typename Vec<u16, 8>::type s8;
    s8 a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = f2bf(v[i]);
    put<FAR>(reinterpret_cast<s8*>(p), a);
  }
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

// The workgroup's sum, in every thread.
__device__ __forceinline__ double group_sum64(double v, double* lds) {
  v = wave_sum64(v);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = 0.0;
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) v += lds[i];
  return v;
}

// f(v, i) of eight elements at a time, v their values, of [from, to); four steps'
// loads are in flight where there are that many.  DOWN: the last ones first.
template <bool DOWN, class T, class F>
__device__ __forceinline__ void clip_each(const T* g, long long from, long long to, F f) {
  const int mine = threadIdx.x * 8;
  auto steps = [&](auto count, long long at) {
    Vec8<T> x[count];
#pragma unroll
    for (int u = 0; u < count; ++u) x[u].load(g + at + u * kChunk + mine);
#pragma unroll
    for (int u = 0; u < count; ++u) f(x[u], at + u * kChunk + mine);
  };
  const std::integral_constant<int, 4> four{};
  const std::integral_constant<int, 1> one{};
  const long long whole = (to - from) / kChunk, fours = whole / 4, rest = from + whole * kChunk;
  auto last = [&] {
    if (rest + mine + 8 <= to) steps(one, rest);
  };
  if (DOWN) {
    last();
    for (long long k = whole; k > fours * 4; --k) steps(one, from + (k - 1) * kChunk);
    for (long long k = fours; k > 0; --k) steps(four, from + (k - 1) * 4 * kChunk);
  } else {
    for (long long k = 0; k < fours; ++k) steps(four, from + k * 4 * kChunk);
    for (long long k = fours * 4; k < whole; ++k) steps(one, from + k * kChunk);
    last();
  }
}
// Elements that are in none of those: fewer than eight, of one thread.
template <class F>
__device__ __forceinline__ void clip_rest(long long from, long long to, F f) {
  const long long at = from + (to - from) / kChunk * kChunk + threadIdx.x * 8;
  if (at < to && at + 8 > to)
    for (long long i = at; i < to; ++i) f(i);
}

template <class T>
__device__ __forceinline__ double clip_squares(const T* g, long long from, long long to) {
  double s[4] = {};   // four sums: one would wait for itself
  clip_each<false>(g, from, to, [&](const Vec8<T>& x, long long) {
    float v[8];
    x.floats(v);
#pragma unroll
    for (int k = 0; k < 8; ++k) s[k & 3] = fma((double)v[k], (double)v[k], s[k & 3]);
  });
  clip_rest(from, to, [&](long long i) {
    const double v = one_float(g[i]);
    s[0] = fma(v, v, s[0]);
  });
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// Workgroup b's share of the sum, a run of chunks, is added to slot b or is its first
// value.  The first workgroup writes the set's part of the table.
__global__ void __launch_bounds__(kThreads) k_clip_norm(ClipSet a, uint32_t total, int written, uint32_t base,
                                                        double* slots, ClipEntry* table) {
  __shared__ double lds[kThreads / 64];
  const int lane = threadIdx.x & 63;
  if (table && blockIdx.x == 0)
    for (int k = threadIdx.x; k < a.count; k += kThreads)
      table[k] = ClipEntry{a.g[k], a.out[k], clip_size(a.n[k]), base + a.end[k],
                           (a.gbf[k >> 5] >> (k & 31) & 1) | (a.obf[k >> 5] >> (k & 31) & 1) << 1};
  if (!slots) return;
  const uint32_t per = (total + gridDim.x - 1) / gridDim.x;
  uint32_t c = blockIdx.x * per;
  const uint32_t stop = min(c + per, total);
  // the gradient of the first chunk: the number of those that end before it
  int k = 0;
#pragma unroll
  for (int i = 0; i < kSet; i += 64)
    k += __popcll(__ballot(i + lane < a.count && a.end[min(i + lane, kSet - 1)] <= c));
  k = __builtin_amdgcn_readfirstlane(k);
  double s = 0.0;
  for (; c < stop; ++k) {
    const uint32_t first = k ? a.end[k - 1] : 0u, last = min(a.end[k], stop);
    const long long from = (long long)(c - first) * kChunk;
    const long long to = min((long long)(last - first) * kChunk, clip_size(a.n[k]));
    s += a.gbf[k >> 5] >> (k & 31) & 1 ? clip_squares((const u16*)a.g[k], from, to)
                                       : clip_squares((const float*)a.g[k], from, to);
    c = last;
  }
  s = group_sum64(s, lds);
  if (threadIdx.x == 0) slots[blockIdx.x] = (int)blockIdx.x < written ? slots[blockIdx.x] + s : s;
}

template <bool FAR, class T, class O>
__device__ __forceinline__ void clip_scale(const T* g, O* out, long long from, long long to, float a, float f) {
  clip_each<true>(g, from, to, [&](const Vec8<T>& x, long long i) {
    float v[8];
    x.floats(v);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = v[k] * a * f;
    store8<FAR>(out + i, v);
  });
  clip_rest(from, to, [&](long long i) {
    const float v = one_float(g[i]) * a * f;
    if constexpr (sizeof(O) == 4) out[i] = v;
    else out[i] = f2bf(v);
  });
}

// Every workgroup adds up the slots by itself, in one order, and scales a run of
// chunks: the last runs first, each from its end on, and on the XCD whose workgroup
// read it for the norm, so that what was read last is found in its cache (12 million
// fp32 gradients in both launches: 30.2 us with runs on any XCD, 28.2 on their own,
// 26.8 from their ends on; 111 million bf16 ones 111.8, 111.6 and 108.3).  A norm that
// is not finite in fp64, as a gradient's infinity or NaN makes it, clips nothing; one
// that only fp32 cannot hold does.
template <bool FAR>
__global__ void __launch_bounds__(kThreads) k_clip_scale(const ClipEntry* table, int count, uint32_t total, int slots_n,
                                                         const double* slots, float scale, float max_norm,
                                                         float* norm_out) {
  __shared__ double lds[kThreads / 64];
  const int lane = threadIdx.x & 63;
  const uint32_t per = (total + gridDim.x - 1) / gridDim.x;
  const uint32_t eights = gridDim.x / 8, b = blockIdx.x;
  const uint32_t start = (b / 8 < eights ? (eights - 1 - b / 8) * 8 + b % 8 : b) * per;
  uint32_t stop = min(start + per, total);
  // the gradient of the last chunk, first among 64 times 64
  const uint32_t c = stop - 1;
  int k = 64 * __popcll(__ballot(64 * lane + 63 < count && table[min(64 * lane + 63, count - 1)].end <= c));
  k += __popcll(__ballot(k + lane < count && table[min(k + lane, count - 1)].end <= c));
  k = __builtin_amdgcn_readfirstlane(k);
  double s = 0.0;
  for (int i = threadIdx.x; i < slots_n; i += kThreads) s += slots[i];
  s = group_sum64(s, lds);
  const double norm = sqrt(s) * fabs((double)scale);
  if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
  const double factor = norm > (double)max_norm && norm < INFINITY ? (double)scale * ((double)max_norm / norm) : scale;
  // a factor that fp32 holds only as a subnormal is two: the first loses nothing
  const float a = fabs(factor) < 0x1p-100 ? 0x1p-64f : 1.f, f = (float)(a == 1.f ? factor : factor * 0x1p64);
  for (; start < stop; --k) {
    const ClipEntry e = table[k];
    const uint32_t first = k ? table[k - 1].end : 0u, at = max(first, start);
    const long long from = (long long)(at - first) * kChunk, to = min((long long)(stop - first) * kChunk, e.n);
    stop = at;
    if (!e.out || (e.out == e.g && factor == 1.0)) continue;
    if (e.types & 1) e.types & 2 ? clip_scale<FAR>((const u16*)e.g, (u16*)e.out, from, to, a, f)
                                 : clip_scale<FAR>((const u16*)e.g, (float*)e.out, from, to, a, f);
    else e.types & 2 ? clip_scale<FAR>((const float*)e.g, (u16*)e.out, from, to, a, f)
                     : clip_scale<FAR>((const float*)e.g, (float*)e.out, from, to, a, f);
  }
}

struct ClipFill {
  ClipSet set;
  uint32_t total;      // its chunks
  long long written;   // elements of the outputs
};
// The next set of gradients from `at` on; returns where the one after it begins.
int clip_fill(const cavs_grad* grads, int count, int at, ClipFill& f) {
  ClipSet& a = f.set;
  a.count = 0;
  f.total = 0;
  f.written = 0;
  std::fill(std::begin(a.gbf), std::end(a.gbf), 0u);
  std::fill(std::begin(a.obf), std::end(a.obf), 0u);
  for (; at < count && a.count < kSet; ++at) {
    const cavs_grad& g = grads[at];
    if (g.n == 0) continue;
    const int k = a.count++;
    a.g[k] = g.g;
    a.out[k] = g.out;
    a.n[k] = (uint32_t)g.n;
    f.total += (uint32_t)((g.n + kChunk - 1) / kChunk);
    if (g.out) f.written += g.n;
    a.end[k] = f.total;
    if (g.g_type == CAVS_T_BF16) a.gbf[k >> 5] |= 1u << (k & 31);
    if (g.out_type == CAVS_T_BF16) a.obf[k >> 5] |= 1u << (k & 31);
  }
  return at;
}

}  // namespace

size_t clip_ws_bytes() { return kSlots * sizeof(double) + kTable * sizeof(ClipEntry); }

cavs_status clip_run(cavs_ctx* ctx, const cavs_grad* grads, int count, float scale, float max_norm, float* norm,
                     void* ws, size_t ws_bytes) {
  if (count < 0 || (count > 0 && !grads)) return fail(ctx, CAVS_ERR_ARG, "bad list of gradients");
  if (!(max_norm >= 0.f)) return fail(ctx, CAVS_ERR_ARG, "max_norm must be at least 0");
  if (!std::isfinite(scale)) return fail(ctx, CAVS_ERR_ARG, "scale must be finite");
  if (!norm) return fail(ctx, CAVS_ERR_ARG, "norm is required");
  for (int i = 0; i < count; ++i) {
    const cavs_grad& g = grads[i];
    auto known = [](int t) { return t == CAVS_T_F32 || t == CAVS_T_BF16; };
    if (!known(g.g_type) || !known(g.out_type)) return fail(ctx, CAVS_ERR_ARG, "gradient %d: unknown element type", i);
    if (g.n < 0 || (g.n > 0 && !g.g)) return fail(ctx, CAVS_ERR_ARG, "gradient %d: bad n or g", i);
    if (g.n > 1ll << 32) return fail(ctx, CAVS_ERR_UNSUPPORTED, "gradient %d: more than 2^32 elements", i);
    if ((uintptr_t)g.g % (g.g_type == CAVS_T_BF16 ? 2 : 4) || (uintptr_t)g.out % (g.out_type == CAVS_T_BF16 ? 2 : 4))
      return fail(ctx, CAVS_ERR_ARG, "gradient %d is not aligned to its elements", i);
    if (g.g == g.out && g.n > 0 && g.g_type != g.out_type)
      return fail(ctx, CAVS_ERR_ARG, "gradient %d: in place, g and out have one type", i);
  }
  if (!ws || ws_bytes < clip_ws_bytes())
    return fail(ctx, CAVS_ERR_WORKSPACE, "workspace too small: %zu < %zu", ws_bytes, clip_ws_bytes());
  if (((uintptr_t)ws & 7) != 0) return fail(ctx, CAVS_ERR_ARG, "ws must be aligned to 8 bytes");
  double* slots = (double*)ws;
  ClipEntry* table = (ClipEntry*)(slots + kSlots);
  ClipFill f;
  // gradients that share a table, their chunks, and elements of their outputs
  struct Round {
    int entries;
    uint32_t chunks;
    long long written;
    void add(const ClipFill& f) {
      entries += f.set.count;
      chunks += f.total;
      written += f.written;
    }
  };
  auto fits = [&](const Round& r) { return r.entries + f.set.count <= kTable && r.chunks + (uint64_t)f.total < 1u << 31; };
  int written = 0;
  Round first{};
  bool open = true;   // the first round takes this set
  int second = count;
  for (int at = 0; at < count;) {
    const int from = at;
    at = clip_fill(grads, count, at, f);
    if (f.total == 0) continue;
    if (open && !fits(first)) {
      open = false;
      second = from;
    }
    const int blocks = (int)std::min<uint32_t>(f.total, kSlots);
    CAVS_LAUNCH("k_clip_norm", k_clip_norm, dim3(blocks), dim3(kThreads), 0, ctx->stream, f.set, f.total, written,
                first.chunks, slots, open ? table + first.entries : nullptr);
    written = std::max(written, blocks);
    if (open) first.add(f);
  }
  auto scaled = [&](const Round& r, float* to) {
    const bool far = r.written >= kFar;
    CAVS_LAUNCH(far ? "k_clip_scale<far>" : "k_clip_scale", far ? k_clip_scale<true> : k_clip_scale<false>,
                dim3(std::max(1u, std::min<uint32_t>(r.chunks, kSlots))), dim3(kThreads), 0, ctx->stream,
                (const ClipEntry*)table, r.entries, r.chunks, written, (const double*)slots, scale, max_norm, to);
  };
  bool any = false;
  for (int i = 0; i < count; ++i) any |= grads[i].out && grads[i].n > 0;
  if (!any) first = Round{};
  scaled(first, norm);
  // what the table could not hold, a table at a time
  for (int at = second; any && at < count;) {
    Round r{};
    while (at < count) {
      const int from = at;
      at = clip_fill(grads, count, at, f);
      if (f.total == 0) continue;
      if (!fits(r)) {
        at = from;
        break;
      }
      CAVS_LAUNCH("k_clip_norm", k_clip_norm, dim3(1), dim3(kThreads), 0, ctx->stream, f.set, f.total, 0, r.chunks,
                  (double*)nullptr, table + r.entries);
      r.add(f);
    }
    scaled(r, nullptr);
  }
  CAVS_LAUNCH_CHECK(ctx);
  return CAVS_OK;
}

}  // namespace cavs
