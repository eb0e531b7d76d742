// Rules on logits: what a model's scores become before the next word is taken.
//
//   v = z_c; said k > 0 times so far: v = v > 0 ? v / r : v r, then v - p, then v - f k
//   v + bias_c + (sum of the row's own biases of c), -inf where the mask's bit is
//   clear, v / T
//
// and of each row the first of its largest v and ln sum exp v.  One pass over the
// logits: bound by memory, the row in and out once.
#include <algorithm>
#include <utility>

#include "vocab.h"

namespace cavs {
namespace {

constexpr int kRulesMaxN = 1 << 20, kRulesMaxC = 1 << 20, kRulesMaxL = 1 << 20, kRulesMaxK = 1024;
// Words of a thread: 16, or 8 where pieces of 16 are too few to have eight on every CU
// (64 x 50 001, every rule: 12.8 us with 16, 11.0 with 8; 256 x 128 000: 32 and 40).
constexpr int kPer = 16, kPerFew = 8;

struct RulesNet {
  int n, C, L, K, M, W32;   // W32 words of 32 bits to a mask
  const float *bias, *repeat, *presence, *frequency, *extra, *temp;
  const int *past, *word, *mask_row;
  const uint32_t* mask;
  int* best;
  float* lse;
  float4* part;   // [n][segments][wavefronts]: largest, sum of exp(v - largest), its word
  int segs;
  int* err;
};

// A largest value and the first word that has it.
struct Top {
  float v;
  int c;
};

// Over the wavefront, in every lane: sixteen lanes by rotation, then the four rows.
template <class F>
__device__ __forceinline__ float wave_all(float v, F f) {
  auto ror = [](float x, auto n) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x120 + decltype(n)::value, 15, 15, true));
  };
  v = f(v, ror(v, std::integral_constant<int, 8>{}));
  v = f(v, ror(v, std::integral_constant<int, 4>{}));
  v = f(v, ror(v, std::integral_constant<int, 2>{}));
  v = f(v, ror(v, std::integral_constant<int, 1>{}));
  auto row = [&](int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l)); };
  return f(f(row(0), row(16)), f(row(32), row(48)));
}
__device__ __forceinline__ Top wave_top(Top t) {
  const float v = wave_all(t.v, [](float x, float y) { return fmaxf(x, y); });
  // words are below 2^20: as floats they are what they are
  const float c = wave_all(t.v == v ? (float)t.c : INFINITY, [](float x, float y) { return fminf(x, y); });
  return Top{v, (int)c};
}
__device__ __forceinline__ float wave_total(float s) {
  return wave_all(s, [](float x, float y) { return x + y; });
}

// A wavefront joins n parts (largest, sum of exp(v - largest), its word) of a row.
__device__ __forceinline__ void rules_join(const RulesNet& a, int row, const float4* part, int n) {
  const int lane = threadIdx.x & 63;
  Top top{-INFINITY, 1 << 20};
  for (int k = lane; k < n; k += 64)   // ascending words
    if (part[k].x > top.v) top = Top{part[k].x, __float_as_int(part[k].z)};
  top = wave_top(top);
  float s = 0.f;
  for (int k = lane; k < n; k += 64)
    // a part without a finite value adds what it has (nothing, or NaN)
    s += fabsf(part[k].x) < INFINITY && fabsf(top.v) < INFINITY
             ? part[k].y * __builtin_amdgcn_exp2f((part[k].x - top.v) * kLog2e) : part[k].y;
  s = wave_total(s);
  if (lane != 0) return;
  if (a.best) a.best[row] = top.v == -INFINITY ? -1 : top.c;
  // all words masked, or the largest is infinite: no sum, unless there is a NaN
  if (a.lse) a.lse[row] = s != s || fabsf(top.v) < INFINITY ? top.v + logf(s) : top.v;
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
// FAR: past the caches.
template <bool FAR, class T, int V>
__device__ __forceinline__ void store_any(T* p, const float (&v)[V]) {
  if constexpr (sizeof(T) == 4) {
    typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      const f4 a = {v[i], v[i + 1], v[i + 2], v[i + 3]};
      if constexpr (FAR) __builtin_nontemporal_store(a, reinterpret_cast<f4*>(p + i));
      else *reinterpret_cast<f4*>(p + i) = a;
    }
  } else {
    typedef uint32_t w __attribute__((ext_vector_type(V / 2), aligned(2)));
    w a;
#pragma unroll
    for (int i = 0; i < V / 2; ++i) a[i] = f2bf2(v[2 * i], v[2 * i + 1]);
    if constexpr (FAR) __builtin_nontemporal_store(a, reinterpret_cast<w*>(p));
    else *reinterpret_cast<w*>(p) = a;
  }
}

// x[at] += e where `here`, at the same for the wavefront: one branch of many.
template <int NV, int V, unsigned... S>
__device__ __forceinline__ void add_at(float (&x)[NV][V], unsigned at, bool here, float e,
                                       std::integer_sequence<unsigned, S...>) {
  (void)((at == S && (x[S / V][S % V] = here ? x[S / V][S % V] + e : x[S / V][S % V], true)) || ...);
}

// A workgroup takes a piece, PER words a thread of one row, a thread vectors of V
// adjacent ones, 16 bytes of the narrower type.  Everything that it reads is asked for
// before anything is waited for.  Counts of the words so far are kept in LDS for the
// piece's words alone; whole numbers, so that no run differs.  Each wavefront leaves
// its largest v and its sum.
// (Workgroups that go through pieces and ask for the next one ahead were slower: 256
// x 128 000 in bf16 49 us, 39 with one for each piece.)
template <class Z, class O, int THREADS, int PER, bool FAR>
__global__ void __launch_bounds__(THREADS) k_rules(RulesNet a, int row0, const Z* z, O* out) {
#pragma clang fp contract(off)
  constexpr int SEG = THREADS * PER, V = sizeof(Z) == 4 && sizeof(O) == 4 ? 4 : 8, NV = PER / V, W = THREADS / 64;
  extern __shared__ uint4 lds[];
  __shared__ float4 parts[W];
  const int tid = threadIdx.x, row = row0 + blockIdx.x / a.segs, c0 = blockIdx.x % a.segs * SEG;
  const int len = min(SEG, a.C - c0);
  uint32_t* count = reinterpret_cast<uint32_t*>(lds);
  typedef Z Raw __attribute__((ext_vector_type(V), aligned(sizeof(Z))));
  Raw raw[NV];
  const Z* zr = z + (size_t)row * a.C + c0;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * THREADS + tid) * V;
    if (c + V <= len) raw[k] = *reinterpret_cast<const Raw*>(zr + c);
  }
  const int* past = a.past + (size_t)row * a.L;
  auto ask = [&](int at, auto& w) {   // a thread's words of the past from `at` on
    int k = 0;
    for (int& x : w) {
      x = at + k < a.L ? past[at + k] : -1;
      k += THREADS;
    }
  };
  int said[2];
  if (a.past) ask(tid, said);
  const int lane = tid & 63;
  int word = -1;       // a wavefront's next 64 of the row's own words, and their biases
  float extra = 0.f;
  auto ask_own = [&](int at) {
    word = at + lane < a.K ? a.word[(size_t)row * a.K + at + lane] : -1;
    extra = at + lane < a.K ? a.extra[(size_t)row * a.K + at + lane] : 0.f;
  };
  if (a.K) ask_own(0);
  const float r = a.repeat ? a.repeat[row] : 1.f, p = a.presence ? a.presence[row] : 0.f;
  const float f = a.frequency ? a.frequency[row] : 0.f, T = a.temp ? a.temp[row] : 1.f;
  uint32_t bits[NV];
  if (a.mask) {
    const int m = a.mask_row ? a.mask_row[row] : a.M == 1 ? 0 : row;
    const bool there = (unsigned)m < (unsigned)a.M;
    if (!there && m != -1 && tid == 0) a.err[1] = 1;
    const uint32_t* mask = a.mask + (size_t)(there ? m : 0) * a.W32 + c0 / 32;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
      const int c = (k * THREADS + tid) * V;
      bits[k] = there && c < len ? mask[c / 32] >> (c % 32) : ~0u;
    }
  }
  bool bad = false;
  if (a.past) {
    for (int i = tid; i < SEG / 4; i += THREADS) lds[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    auto count_in = [&](const auto& words) {
      for (const int w : words) {
        if ((unsigned)(w - c0) < (unsigned)len) atomicAdd(&count[w - c0], 1u);
        bad |= (unsigned)(w + 1) > (unsigned)a.C;
      }
    };
    count_in(said);
    for (int at = 2 * THREADS; at < a.L; at += 8 * THREADS) {
      int more[8];
      ask(at + tid, more);
      count_in(more);
    }
    __syncthreads();
  }
  // The row's own biases: each wavefront looks for those of its words and adds them up,
  // in the list's order, in the registers of the lane that has the word.  (Through a
  // table of the piece's words in LDS, 126 x 130 000 with 64 of them took 45 us, 24
  // without any.)
  float own[NV][V];
  if (a.K) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) own[k][i] = 0.f;
    for (int at = 0; at < a.K; at += 64) {
      const int c = word - c0;
      const float e = extra;
      bad |= (unsigned)(word + 1) > (unsigned)a.C;
      unsigned long long mine =
          __ballot((unsigned)c < (unsigned)len && (unsigned)c / V % THREADS / 64 == (unsigned)tid / 64);
      if (at + 64 < a.K) ask_own(at + 64);
      while (mine) {
        const int l = __ffsll(mine) - 1;
        mine &= mine - 1;
        const unsigned cl = __builtin_amdgcn_readlane(c, l);
        const float el = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(e), l));
        const bool here = lane == (int)(cl / V % 64);
        const unsigned slot = cl / V / THREADS * V + cl % V;
        add_at(own, slot, here, el, std::make_integer_sequence<unsigned, PER>{});
      }
    }
  }
  if (bad) a.err[1] = 1;
  float v[NV][V];
  Top top{-INFINITY, 1 << 20};
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    const int c = (k * THREADS + tid) * V;
    float(&x)[V] = v[k];
    const bool whole = c + V <= len;
    if (whole) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        if constexpr (sizeof(Z) == 4) x[i] = raw[k][i];
        else x[i] = __uint_as_float((uint32_t)raw[k][i] << 16);
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        x[i] = -INFINITY;
        if (c + i < len) {
          if constexpr (sizeof(Z) == 4) x[i] = zr[c + i];
          else x[i] = __uint_as_float((uint32_t)zr[c + i] << 16);
        }
      }
      if (c >= len) continue;
    }
    if (a.past) {
      uint32_t n[V], any = 0;
#pragma unroll
      for (int i = 0; i < V; i += 4) {
        const uint4 y = *reinterpret_cast<const uint4*>(count + c + i);
        n[i] = y.x, n[i + 1] = y.y, n[i + 2] = y.z, n[i + 3] = y.w;
        any |= y.x | y.y | y.z | y.w;
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
      for (int i = 0; i < V; ++i) x[i] = x[i] + own[k][i];
    if (a.mask)
#pragma unroll
      for (int i = 0; i < V; ++i) x[i] = bits[k] >> i & 1u ? x[i] : -INFINITY;
    if (a.temp)
#pragma unroll
      for (int i = 0; i < V; ++i) x[i] = x[i] / T;
    if (out) {
      O* o = out + (size_t)row * a.C + c0 + c;
      if (whole) {
        store_any<FAR, O, V>(o, x);
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
      sum += x[i] != x[i] ? x[i] : 0.f;
    }
  }
  if (!a.best && !a.lse) return;
  top = wave_top(top);
  if (fabsf(top.v) < INFINITY)
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) sum += __builtin_amdgcn_exp2f((v[k][i] - top.v) * kLog2e);
  sum = wave_total(sum);
  const float4 mine = make_float4(top.v, sum, __int_as_float(top.c), 0.f);
  if (a.segs > 1) {
    if ((tid & 63) == 0) a.part[((size_t)row * a.segs + c0 / SEG) * W + tid / 64] = mine;
  } else {
    if ((tid & 63) == 0) parts[tid / 64] = mine;
    __syncthreads();
    if (tid < 64) rules_join(a, row, parts, W);
  }
}

__global__ void __launch_bounds__(64) k_rules_join(RulesNet a, int n) {
  rules_join(a, blockIdx.x, a.part + (size_t)blockIdx.x * n, n);
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
  return std::max<size_t>(256, (size_t)n * cdiv(C, 256 * kPerFew) * 4 * sizeof(float4));
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
  const bool wide = r->C <= 1024 * kPer && r->C > 256 * kPer;
  const int threads = wide ? 1024 : 256;
  const bool few = !wide && (long)r->n * cdiv(r->C, 256 * kPer) < 2048 && r->C > 256 * kPer;
  const int per = few ? kPerFew : kPer;
  a.segs = cdiv(r->C, threads * per);
  a.err = ctx->dev_err_dev;
  // what is read next does not find 32 MB in the caches (256 x 128 000 in bf16: 32 us
  // through them, 29 past them)
  const bool far = (size_t)r->n * r->C * os >= 32u << 20;
  if (best || lse) {
    if (!ws || ws_bytes < need) return fail(ctx, CAVS_ERR_WORKSPACE, "workspace too small: %zu < %zu", ws_bytes, need);
    if (((uintptr_t)ws & 15) != 0) return fail(ctx, CAVS_ERR_ARG, "ws must be aligned to 16 bytes");
  }
  const size_t shmem = a.past ? (size_t)threads * per * 4 : 0;
  // a launch has fewer than 2^32 threads
  const int step = std::max(1, (int)std::min<long>(r->n, (1l << 30) / threads / a.segs));
  for (int i = 0; i < r->n; i += step) {
    const dim3 grid((unsigned)std::min(step, r->n - i) * a.segs);
    auto go = [&](auto zt, auto ot) {
      using Z = decltype(zt);
      using O = decltype(ot);
      auto launch = [&](const char* name, auto kernel) {
        CAVS_LAUNCH(name, kernel, grid, dim3(threads), shmem, ctx->stream, a, i, (const Z*)z, (O*)out);
      };
      if (wide) launch("k_rules<1024, 16>", k_rules<Z, O, 1024, kPer, false>);
      else if (few) launch("k_rules<256, 8>", k_rules<Z, O, 256, kPerFew, false>);
      else if (far) launch("k_rules<256, 16, far>", k_rules<Z, O, 256, kPer, true>);
      else launch("k_rules<256, 16>", k_rules<Z, O, 256, kPer, false>);
    };
    if (zs == 2) os == 2 ? go(u16{}, u16{}) : go(u16{}, float{});
    else os == 2 ? go(float{}, u16{}) : go(float{}, float{});
  }
  if ((best || lse) && a.segs > 1)
    CAVS_LAUNCH("k_rules_join", k_rules_join, dim3(r->n), dim3(64), 0, ctx->stream, a, 4 * a.segs);
  CAVS_LAUNCH_CHECK(ctx);
  return CAVS_OK;
}

}  // namespace cavs
