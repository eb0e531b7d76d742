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

#include "vocab.h"

namespace cavs {
namespace {

constexpr int kSlots = 1024;    // workgroups of a launch, each with a partial sum
constexpr int kSet = 120;       // gradients of a launch: their list is its argument
constexpr int kChunk = 8192;    // elements that a workgroup takes at a time

// Gradients of a launch; chunks[k] is the number of chunks up to and with the k-th.
struct ClipSet {
  const void* g[kSet];
  void* out[kSet];
  long long n[kSet];
  uint32_t chunks[kSet];
  uint32_t gbf[(kSet + 31) / 32], obf[(kSet + 31) / 32];
  int count;
};
static_assert(sizeof(ClipSet) <= 3584, "kernel arguments");

// Vectors at any address that is aligned to its elements.
template <class T, int V>
struct Vec {
  typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T))));
};

template <class T>
__device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
    typedef typename Vec<float, 4>::type f4;
    const f4 a = *reinterpret_cast<const f4*>(p), b = *reinterpret_cast<const f4*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
  } else {
    typedef typename Vec<u16, 8>::type s8;
    const s8 a = *reinterpret_cast<const s8*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float((uint32_t)a[i] << 16);
  }
}
template <class T>
__device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
  if constexpr (sizeof(T) == 4) {
    typedef typename Vec<float, 4>::type f4;
    *reinterpret_cast<f4*>(p) = f4{v[0], v[1], v[2], v[3]};
    *reinterpret_cast<f4*>(p + 4) = f4{v[4], v[5], v[6], v[7]};
  } else {
    typedef typename Vec<u16, 8>::type s8;
    s8 a;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = f2bf(v[i]);
    *reinterpret_cast<s8*>(p) = a;
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
  __syncthreads();
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// The gradient that a chunk belongs to: the number of those that end before it.
__device__ __forceinline__ int clip_owner(const ClipSet& a, uint32_t chunk) {
  const int lane = threadIdx.x & 63;
  const bool b0 = lane < a.count && a.chunks[lane] <= chunk;
  const bool b1 = 64 + lane < a.count && a.chunks[min(64 + lane, kSet - 1)] <= chunk;
  return __popcll(__ballot(b0)) + __popcll(__ballot(b1));
}

template <class T>
__device__ __forceinline__ double clip_squares(const T* g, int n) {
  double s = 0.0;
  for (int i = threadIdx.x * 8; i < n; i += 256 * 8) {
    if (i + 8 <= n) {
      float v[8];
      load8(g + i, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) s = fma((double)v[k], (double)v[k], s);
    } else {
      for (int k = i; k < n; ++k) {
        float v;
        if constexpr (sizeof(T) == 4) v = g[k];
        else v = __uint_as_float((uint32_t)g[k] << 16);
        s = fma((double)v, (double)v, s);
      }
    }
  }
  return s;
}

// Workgroup b's share of the sum is added to slot b, or is its first value.
__global__ void __launch_bounds__(256) k_clip_norm(ClipSet a, uint32_t total, int written, double* slots) {
  __shared__ double lds[4];
  double s = 0.0;
  for (uint32_t chunk = blockIdx.x; chunk < total; chunk += gridDim.x) {
    const int k = __builtin_amdgcn_readfirstlane(clip_owner(a, chunk));
    const long long at = (long long)(chunk - (k ? a.chunks[k - 1] : 0u)) * kChunk;
    const int n = (int)min((long long)kChunk, a.n[k] - at);
    s += a.gbf[k >> 5] >> (k & 31) & 1 ? clip_squares((const u16*)a.g[k] + at, n)
                                       : clip_squares((const float*)a.g[k] + at, n);
  }
  s = group_sum64(s, lds);
  if (threadIdx.x == 0) slots[blockIdx.x] = (int)blockIdx.x < written ? slots[blockIdx.x] + s : s;
}

template <class T, class O>
__device__ __forceinline__ void clip_scale(const T* g, O* out, int n, float a, float f) {
  for (int i = threadIdx.x * 8; i < n; i += 256 * 8) {
    if (i + 8 <= n) {
      float v[8];
      load8(g + i, v);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = v[k] * a * f;
      store8(out + i, v);
    } else {
      for (int k = i; k < n; ++k) {
        float v;
        if constexpr (sizeof(T) == 4) v = g[k];
        else v = __uint_as_float((uint32_t)g[k] << 16);
        if constexpr (sizeof(O) == 4) out[k] = v * a * f;
        else out[k] = f2bf(v * a * f);
      }
    }
  }
}

// Every workgroup adds up the slots by itself, in one order.  A norm that is not
// finite clips nothing.
__global__ void __launch_bounds__(256) k_clip_scale(ClipSet a, uint32_t total, int slots_n, const double* slots,
                                                    float scale, float max_norm, float* norm_out) {
  __shared__ double lds[4];
  double s = 0.0;
  for (int i = threadIdx.x; i < slots_n; i += 256) s += slots[i];
  s = group_sum64(s, lds);
  const double norm = sqrt(s) * fabs((double)scale);
  if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
  const double factor = norm > (double)max_norm && norm < INFINITY ? (double)scale * ((double)max_norm / norm) : scale;
  // a factor that fp32 holds only as a subnormal is two: the first loses nothing
  const float a2 = fabs(factor) < 0x1p-100 ? 0x1p-64f : 1.f, f = (float)(a2 == 1.f ? factor : factor * 0x1p64);
  for (uint32_t chunk = blockIdx.x; chunk < total; chunk += gridDim.x) {
    const int k = __builtin_amdgcn_readfirstlane(clip_owner(a, chunk));
    const long long at = (long long)(chunk - (k ? a.chunks[k - 1] : 0u)) * kChunk;
    const int n = (int)min((long long)kChunk, a.n[k] - at);
    const bool gb = a.gbf[k >> 5] >> (k & 31) & 1, ob = a.obf[k >> 5] >> (k & 31) & 1;
    if (a.out[k] == a.g[k] && factor == 1.0) continue;
    if (gb) ob ? clip_scale((const u16*)a.g[k] + at, (u16*)a.out[k] + at, n, a2, f)
               : clip_scale((const u16*)a.g[k] + at, (float*)a.out[k] + at, n, a2, f);
    else ob ? clip_scale((const float*)a.g[k] + at, (u16*)a.out[k] + at, n, a2, f)
            : clip_scale((const float*)a.g[k] + at, (float*)a.out[k] + at, n, a2, f);
  }
}

struct ClipFill {
  ClipSet set;
  uint32_t total;
};
// The next set of gradients from `at` on; out: only those that are written.
int clip_fill(const cavs_grad* grads, int count, int at, bool out, ClipFill& f) {
  ClipSet& a = f.set;
  a.count = 0;
  f.total = 0;
  for (uint32_t& w : a.gbf) w = 0;
  for (uint32_t& w : a.obf) w = 0;
  for (; at < count && a.count < kSet; ++at) {
    const cavs_grad& g = grads[at];
    if (g.n == 0 || (out && !g.out)) continue;
    const int k = a.count++;
    a.g[k] = g.g;
    a.out[k] = g.out;
    a.n[k] = g.n;
    f.total += (uint32_t)((g.n + kChunk - 1) / kChunk);
    a.chunks[k] = f.total;
    if (g.g_type == CAVS_T_BF16) a.gbf[k >> 5] |= 1u << (k & 31);
    if (g.out_type == CAVS_T_BF16) a.obf[k >> 5] |= 1u << (k & 31);
  }
  return at;
}

}  // namespace

size_t clip_ws_bytes() { return kSlots * sizeof(double); }

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
  int written = 0;
  ClipFill f;
  for (int at = 0; at < count;) {
    at = clip_fill(grads, count, at, false, f);
    if (f.total == 0) continue;
    const int blocks = (int)std::min<uint32_t>(f.total, kSlots);
    CAVS_LAUNCH("k_clip_norm", k_clip_norm, dim3(blocks), dim3(256), 0, ctx->stream, f.set, f.total, written, slots);
    written = std::max(written, blocks);
  }
  int at = 0;
  for (bool first = true; first || at < count; first = false) {
    at = clip_fill(grads, count, at, true, f);
    if (!first && f.total == 0) continue;
    CAVS_LAUNCH("k_clip_scale", k_clip_scale, dim3(std::max(1u, std::min<uint32_t>(f.total, 2 * kSlots))), dim3(256), 0,
                ctx->stream, f.set, f.total, written, (const double*)slots, scale, max_norm, first ? norm : nullptr);
  }
  CAVS_LAUNCH_CHECK(ctx);
  return CAVS_OK;
}

}  // namespace cavs
