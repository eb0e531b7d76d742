// Rules on logits: what a model's scores become before the next word is taken.
//
//   v = z_c; said k > 0 times so far: v = v > 0 ? v / r : v r, then v - p, then v - f k
//   v + bias_c + (sum of the row's own biases of c), -inf where the mask's bit is
//   clear, v / T
//
// and of each row the first of its largest v and ln sum exp v.  One pass over the
// logits: bound by memory, the row in and out once.
#include <algorithm>

#include "vocab.h"

namespace cavs {
namespace {

constexpr int kRulesMaxN = 1 << 20, kRulesMaxC = 1 << 20, kRulesMaxL = 1 << 20, kRulesMaxK = 1024;
constexpr int kPer = 16;   // words of a thread

struct RulesNet {
  int n, C, L, K, M, W32;   // W32 words of 32 bits to a mask
  const float *bias, *repeat, *presence, *frequency, *extra, *temp;
  const int *past, *word, *mask_row;
  const uint32_t* mask;
  int* best;
  float* lse;
  float4* part;   // [n][segments]: largest, sum of exp(v - largest), its word
  int segs;
  int* err;
};

// Largest value and its first word, over the workgroup.
struct Top {
  float v;
  int c;
};
__device__ __forceinline__ Top higher(Top a, Top b) {
  return b.v > a.v || (b.v == a.v && b.c < a.c) ? b : a;
}
__device__ __forceinline__ Top wave_top(Top t) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) t = higher(t, Top{__shfl_xor(t.v, o, kWave), __shfl_xor(t.c, o, kWave)});
  return t;
}

__device__ __forceinline__ void rules_write(const RulesNet& a, int row, Top t, float sum) {
  // sum is of exp(v - t.v); all words masked, or the largest is infinite: no sum
  if (a.best) a.best[row] = t.v == -INFINITY ? -1 : t.c;
  if (a.lse) a.lse[row] = sum != sum || fabsf(t.v) < INFINITY ? t.v + logf(sum) : t.v;
}

// V adjacent elements at any address that is aligned to them.
template <class T, int V>
__device__ __forceinline__ void load_any(const T* p, float (&v)[V]) {
  if constexpr (sizeof(T) == 4) {
    typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const f4 a = *reinterpret_cast<const f4*>(p + i);
      v[i] = a[0], v[i + 1] = a[1], v[i + 2] = a[2], v[i + 3] = a[3];
    }
  } else {
    typedef u16 s __attribute__((ext_vector_type(V), aligned(2)));
    const s a = *reinterpret_cast<const s*>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = __uint_as_float((uint32_t)a[i] << 16);
  }
}
template <class T, int V>
__device__ __forceinline__ void store_any(T* p, const float (&v)[V]) {
  if constexpr (sizeof(T) == 4) {
    typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
    for (int i = 0; i < V; i += 4) *reinterpret_cast<f4*>(p + i) = f4{v[i], v[i + 1], v[i + 2], v[i + 3]};
  } else {
    typedef uint32_t w __attribute__((ext_vector_type(V / 2), aligned(2)));
    w a;
#pragma unroll
    for (int i = 0; i < V / 2; ++i) a[i] = f2bf2(v[2 * i], v[2 * i + 1]);
    *reinterpret_cast<w*>(p) = a;
  }
}

// A workgroup takes kPer words a thread of one row, in pieces of V adjacent ones, 16
// bytes of the narrower type.  Counts of the words so far and sums of the row's own
// biases are kept in LDS for its words alone; whole numbers and a fixed order, so
// that no run differs.
template <class Z, class O, int THREADS>
__global__ void __launch_bounds__(THREADS) k_rules(RulesNet a, int row0, const Z* z, O* out) {
#pragma clang fp contract(off)
  constexpr int SEG = THREADS * kPer, V = sizeof(Z) == 4 && sizeof(O) == 4 ? 4 : 8, NV = kPer / V;
  extern __shared__ uint4 lds[];
  __shared__ Top tops[THREADS / 64];
  __shared__ float sums[THREADS / 64];
  const int tid = threadIdx.x, row = row0 + blockIdx.x / a.segs, seg = blockIdx.x % a.segs;
  const int c0 = seg * SEG, len = min(SEG, a.C - c0);
  uint32_t* count = reinterpret_cast<uint32_t*>(lds);
  float* own = reinterpret_cast<float*>(lds + (a.past ? SEG / 4 : 0));
  float v[NV][V];
  const Z* zr = z + (size_t)row * a.C + c0;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * THREADS + tid) * V;
    if (c + V <= len) {
      load_any<Z, V>(zr + c, v[k]);
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        v[k][i] = -INFINITY;
        if (c + i < len) {
          if constexpr (sizeof(Z) == 4) v[k][i] = zr[c + i];
          else v[k][i] = __uint_as_float((uint32_t)zr[c + i] << 16);
        }
      }
    }
  }
  if (a.past || a.K) {
    for (int i = tid; i < ((a.past ? SEG : 0) + (a.K ? SEG : 0)) / 4; i += THREADS) lds[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    bool bad = false;
    if (a.past)
      for (int i = tid; i < a.L; i += THREADS) {
        const int w = a.past[(size_t)row * a.L + i];
        if ((unsigned)(w - c0) < (unsigned)len) atomicAdd(&count[w - c0], 1u);
        bad |= (unsigned)(w + 1) > (unsigned)a.C;
      }
    if (a.K) {
      const int* word = a.word + (size_t)row * a.K;
      const float* extra = a.extra + (size_t)row * a.K;
      for (int i = tid; i < a.K; i += THREADS) {
        const int w = word[i];
        bad |= (unsigned)(w + 1) > (unsigned)a.C;
        if ((unsigned)(w - c0) >= (unsigned)len) continue;
        // the first of a word's places adds all of them
        bool first = true;
        for (int j = 0; j < i; ++j) first &= word[j] != w;
        if (!first) continue;
        float s = extra[i];
        for (int j = i + 1; j < a.K; ++j)
          if (word[j] == w) s += extra[j];
        own[w - c0] = s;
      }
    }
    if (bad && seg == 0) a.err[1] = 1;
    __syncthreads();
  }
  const float r = a.repeat ? a.repeat[row] : 1.f, p = a.presence ? a.presence[row] : 0.f;
  const float f = a.frequency ? a.frequency[row] : 0.f, T = a.temp ? a.temp[row] : 1.f;
  const uint32_t* mask = nullptr;
  if (a.mask) {
    const int m = a.mask_row ? a.mask_row[row] : a.M == 1 ? 0 : row;
    if ((unsigned)m < (unsigned)a.M) mask = a.mask + (size_t)m * a.W32 + c0 / 32;
    else if (m != -1 && tid == 0 && seg == 0) a.err[1] = 1;
  }
  Top top{-INFINITY, 0x7fffffff};
  float nan = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * THREADS + tid) * V;
    if (c >= len) continue;
    float(&x)[V] = v[k];
    if (a.past) {
      uint32_t n[V], any = 0;
#pragma unroll
      for (int i = 0; i < V; i += 4) {
        const uint4 q = *reinterpret_cast<const uint4*>(count + c + i);
        n[i] = q.x, n[i + 1] = q.y, n[i + 2] = q.z, n[i + 3] = q.w;
        any |= q.x | q.y | q.z | q.w;
      }
      if (any)
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (n[i]) {
            x[i] = x[i] > 0.f ? x[i] / r : x[i] * r;
            x[i] = x[i] - p;
            x[i] = x[i] - f * (float)n[i];
          }
    }
    const bool whole = c + V <= len;
    if (a.bias) {
      const float* b = a.bias + c0 + c;
      float y[V];
      if (whole) {
        load_any<float, V>(b, y);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = c + i < len ? b[i] : 0.f;
      }
#pragma unroll
      for (int i = 0; i < V; ++i) x[i] = x[i] + y[i];
    }
    if (a.K)
#pragma unroll
      for (int i = 0; i < V; i += 4) {
        const float4 q = *reinterpret_cast<const float4*>(own + c + i);
        x[i] = x[i] + q.x, x[i + 1] = x[i + 1] + q.y, x[i + 2] = x[i + 2] + q.z, x[i + 3] = x[i + 3] + q.w;
      }
    if (mask) {
      const uint32_t bits = mask[c / 32] >> (c % 32);
#pragma unroll
      for (int i = 0; i < V; ++i) x[i] = bits >> i & 1u ? x[i] : -INFINITY;
    }
    if (a.temp)
#pragma unroll
      for (int i = 0; i < V; ++i) x[i] = x[i] / T;
    if (out) {
      O* o = out + (size_t)row * a.C + c0 + c;
      if (whole) {
        store_any<O, V>(o, x);
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
          if (c + i < len) {
            if constexpr (sizeof(O) == 4) o[i] = x[i];
            else o[i] = f2bf(x[i]);
          }
      }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (!whole && c + i >= len) x[i] = -INFINITY;
      if (x[i] > top.v) top = Top{x[i], c0 + c + i};   // ascending words: the first one stays
      nan += x[i] != x[i] ? x[i] : 0.f;
    }
  }
  if (!a.best && !a.lse) return;
  top = wave_top(top);
  if ((tid & 63) == 0) tops[tid >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < THREADS / 64; ++k) top = higher(top, tops[k]);
  float s = nan;
  if (fabsf(top.v) < INFINITY)
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) s += __builtin_amdgcn_exp2f((v[k][i] - top.v) * kLog2e);
  s = wave_sum(s);
  if ((tid & 63) == 0) sums[tid >> 6] = s;
  __syncthreads();
  if (tid == 0) {
    s = 0.f;
    for (int k = 0; k < THREADS / 64; ++k) s += sums[k];
    if (a.segs == 1) rules_write(a, row, top, s);
    else a.part[(size_t)row * a.segs + seg] = make_float4(top.v, s, __int_as_float(top.c), 0.f);
  }
}

// A wavefront joins a row's segments.
__global__ void __launch_bounds__(64) k_rules_join(RulesNet a, int row0) {
  const int row = row0 + blockIdx.x, lane = threadIdx.x;
  const float4* part = a.part + (size_t)row * a.segs;
  Top top{-INFINITY, 0x7fffffff};
  for (int k = lane; k < a.segs; k += 64) top = higher(top, Top{part[k].x, __float_as_int(part[k].z)});
  top = wave_top(top);
  float s = 0.f;
  for (int k = lane; k < a.segs; k += 64)
    // a segment without a finite word adds what it has (nothing, or NaN)
    s += fabsf(part[k].x) < INFINITY && fabsf(top.v) < INFINITY
             ? part[k].y * __builtin_amdgcn_exp2f((part[k].x - top.v) * kLog2e) : part[k].y;
  s = wave_sum(s);
  if (lane == 0) rules_write(a, row, top, s);
}

cavs_status rules_args(cavs_ctx* ctx, const cavs_rules* r) {
  if (!r) return fail(ctx, CAVS_ERR_ARG, "null rules");
  if ((r->z_type != CAVS_T_F32 && r->z_type != CAVS_T_BF16) ||
      (r->out_type != CAVS_T_F32 && r->out_type != CAVS_T_BF16))
    return fail(ctx, CAVS_ERR_ARG, "unknown element type");
  if (r->n < 0 || r->C <= 0 || r->L < 0 || r->K < 0 || r->M < 0) return fail(ctx, CAVS_ERR_ARG, "bad n/C/L/K/M");
  if (r->n > kRulesMaxN || r->C > kRulesMaxC || r->L > kRulesMaxL || r->K > kRulesMaxK)
    return fail(ctx, CAVS_ERR_UNSUPPORTED, "n=%d, C=%d, L=%d, K=%d: at most %d, %d, %d, %d", r->n, r->C, r->L,
                r->K, kRulesMaxN, kRulesMaxC, kRulesMaxL, kRulesMaxK);
  return CAVS_OK;
}

}  // namespace

size_t adjust_ws_bytes(int n, int C) {
  if (n < 0 || C <= 0 || n > kRulesMaxN || C > kRulesMaxC) return 0;
  return std::max<size_t>(256, (size_t)n * cdiv(C, 256 * kPer) * sizeof(float4));
}

cavs_status adjust_run(cavs_ctx* ctx, const cavs_rules* r, const void* z, void* out, int* best, float* lse,
                       void* ws, size_t ws_bytes) {
  cavs_status st = rules_args(ctx, r);
  if (st != CAVS_OK) return st;
  const int zs = r->z_type == CAVS_T_BF16 ? 2 : 4, os = r->out_type == CAVS_T_BF16 ? 2 : 4;
  if ((r->repeat || r->presence || r->frequency) && r->L > 0 && !r->past)
    return fail(ctx, CAVS_ERR_ARG, "penalties need the words so far");
  if (r->K > 0 && (!r->extra_word || !r->extra)) return fail(ctx, CAVS_ERR_ARG, "extra_word and extra go together");
  if (r->mask && (r->M <= 0 || (!r->mask_row && r->M != 1 && r->M != r->n)))
    return fail(ctx, CAVS_ERR_ARG, "M=%d masks for n=%d rows without mask_row", r->M, r->n);
  if (r->mask_row && !r->mask) return fail(ctx, CAVS_ERR_ARG, "mask_row without masks");
  if (r->n == 0) return CAVS_OK;
  if (!z) return fail(ctx, CAVS_ERR_ARG, "z is required");
  if (!out && !best && !lse) return fail(ctx, CAVS_ERR_ARG, "nothing to write");
  if ((uintptr_t)z % zs || (uintptr_t)out % os) return fail(ctx, CAVS_ERR_ARG, "z or out is not aligned to its elements");
  if (out == z && r->z_type != r->out_type) return fail(ctx, CAVS_ERR_ARG, "in place, z and out have one type");
  const size_t need = adjust_ws_bytes(r->n, r->C);
  RulesNet a{r->n, r->C, r->L, r->K, r->M, cdiv(r->C, 32)};
  a.bias = r->bias;
  a.repeat = r->repeat;
  a.presence = r->presence;
  a.frequency = r->frequency;
  a.extra = r->extra;
  a.temp = r->temp;
  a.past = r->L > 0 && (r->repeat || r->presence || r->frequency) ? r->past : nullptr;
  a.word = r->extra_word;
  a.mask = r->mask;
  a.mask_row = r->mask_row;
  a.best = best;
  a.lse = lse;
  a.part = (float4*)ws;
  // a row of up to 16 384 words in one workgroup, without a join
  const bool wide = r->C <= 1024 * kPer && r->C > 256 * kPer && !(a.past && a.K);
  a.segs = cdiv(r->C, (wide ? 1024 : 256) * kPer);
  a.err = ctx->dev_err_dev;
  if ((best || lse) && a.segs > 1) {
    if (!ws || ws_bytes < need) return fail(ctx, CAVS_ERR_WORKSPACE, "workspace too small: %zu < %zu", ws_bytes, need);
    if (((uintptr_t)ws & 15) != 0) return fail(ctx, CAVS_ERR_ARG, "ws must be aligned to 16 bytes");
  }
  const int threads = wide ? 1024 : 256;
  const size_t shmem = (size_t)threads * kPer * 4 * ((a.past ? 1 : 0) + (a.K ? 1 : 0));
  // a launch has fewer than 2^32 threads
  const int step = std::max(1, (int)std::min<long>(r->n, (1l << 30) / threads / a.segs));
  for (int i = 0; i < r->n; i += step) {
    const dim3 grid((unsigned)std::min(step, r->n - i) * a.segs);
    auto go = [&](auto zt, auto ot) {
      using Z = decltype(zt);
      using O = decltype(ot);
      if (wide)
        CAVS_LAUNCH("k_rules<1024>", (k_rules<Z, O, 1024>), grid, dim3(1024), shmem, ctx->stream, a, i, (const Z*)z, (O*)out);
      else
        CAVS_LAUNCH("k_rules<256>", (k_rules<Z, O, 256>), grid, dim3(256), shmem, ctx->stream, a, i, (const Z*)z, (O*)out);
    };
    if (zs == 2) os == 2 ? go(u16{}, u16{}) : go(u16{}, float{});
    else os == 2 ? go(float{}, u16{}) : go(float{}, float{});
  }
  if ((best || lse) && a.segs > 1)
    CAVS_LAUNCH("k_rules_join", k_rules_join, dim3(r->n), dim3(64), 0, ctx->stream, a, 0);
  CAVS_LAUNCH_CHECK(ctx);
  return CAVS_OK;
}

}  // namespace cavs
