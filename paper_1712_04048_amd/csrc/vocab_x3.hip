// fp32 products of the vocabulary head, on the split products of x3_gemm.h.
#include <algorithm>

#include "vocab.h"
#include "x3_gemm.h"

namespace cavs {
namespace {

// The live rows as a product's columns (tx), rows (ty) or contraction.
struct LiveCols {
  const int* live;
  __device__ void operator()(int& ty, int& tx, int&, int& items) const {
    tx = cdiv_dev(*live, kX3Tile);
    items = tx * ty;
  }
};
struct LiveRows {
  const int* live;
  int S;
  __device__ void operator()(int& ty, int& tx, int&, int& items) const {
    ty = cdiv_dev(*live, kX3Tile);
    items = tx * ty * S;
  }
};
struct LiveK {
  const int* live;
  __device__ void operator()(int&, int&, int& K, int&) const { K = min(K, (*live + 3) & ~3); }
};

// W_s of a C that is no multiple of 4: its quads are loaded at the alignment of a
// float, one that reaches past a row's end an element at a time (the next row's
// values, or none behind the last row, must not meet zeros of the other operand).
// 3 to 5 % of the products' time; a padded copy took 72 of 330 us of 64 rows, 50
// 001 words, H = 1024.
__device__ __forceinline__ float4 load4_upto(const float* p, int there) {
  float4 x = f4zero();
  if (there >= 4) {
    __builtin_memcpy(&x, p, 16);
  } else {
    if (there > 0) x.x = p[0];
    if (there > 1) x.y = p[1];
    if (there > 2) x.z = p[2];
  }
  return x;
}
struct X3WRows : X3Rows {
  __device__ void load(const Net&, const State& s, int k0, int kend, float4 (&v)[8]) const {
    const int k = k0 + 8 * s.q;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        v[2 * j + h] = load4_upto(s.p[j] ? s.p[j] + k0 + 4 * h : nullptr, s.p[j] ? kend - k - 4 * h : 0);
  }
};
struct X3WCols : X3Cols {
  struct State : X3Cols::State {
    int there;
  };
  __device__ void init(const Net& n, State& s, int t, int r0) const {
    X3Cols::init(n, s, t, r0);
    s.there = cols - (r0 + 4 * s.i);
  }
  __device__ void load(const Net&, const State& s, int k0, int kend, float4 (&v)[8]) const {
    const int k = k0 + 8 * s.q;
#pragma unroll
    for (int e = 0; e < 8; ++e)
      v[e] = load4_upto(s.p ? s.p + (k + e) * s.ld : nullptr, k + e < kend ? s.there : 0);
  }
};

template <class L>
struct X3Whole : L {};   // the same braces for whole quads

// Words are the tile's rows: lane (r, g) holds words 64 wm + 16 g + 4 e + j of
// rows 64 wn + 4 r + c.
template <bool LOSS, bool TEACH>
struct X3Vocab {
  VocabEp e;
  __device__ void operator()(const Net&, int, int m0, int n0, int wm, int wn, int g, int r,
                             const v4f (&acc)[4][4]) const {
    const int a0 = e.col0 + m0 + 64 * wm, row0 = n0 + 64 * wn;
    auto col = [](int i, int gg) { return 16 * gg + i; };
    float b[16], db[16] = {};
    vocab_bias(e, a0, g, col, b);
    const int live = *e.live;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      float z[16];
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int j = 0; j < 4; ++j) z[4 * q + j] = acc[j][c][q] + b[4 * q + j];
      const int row = row0 + c + 4 * r;
      vocab_rows16<LOSS, TEACH, float, 64>(e, z, col, row, vocab_row<LOSS, TEACH>(e, row, a0 / 64, live), a0,
                                           (size_t)(a0 / 64) * e.rows + row, db);
    }
    if (!LOSS) vocab_db<64>(e, db, col, a0, row0 / 64);
  }
};

struct X3VocabOut {
  VocabOut o;
  __device__ void operator()(const Net&, int z, int m0, int n0, int wm, int wn, int g, int r,
                             const v4f (&acc)[4][4]) const {
    const int nc = n0 + 64 * wn + 4 * r;
    const float w = o.scale ? *o.scale : 1.f;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        vocab_store4(o, w, z, m0 + 64 * wm + 16 * g + 4 * e + j, nc,
                     make_float4(acc[j][0][e], acc[j][1][e], acc[j][2][e], acc[j][3][e]));
  }
};

Net zero_net(const VocabNet& v) {
  Net n{};
  n.zrow = v.zrow;
  return n;
}

template <bool LOSS, class W>
void logits(const char* name, const VocabNet& v, int col0, int cols, hipStream_t s) {
  const W w{{(const float*)v.Ws + col0, v.ldw, v.C - col0}};
  const X3Rows h{(const float*)v.hp, v.H, v.rows};
  const VocabEp e = vocab_ep(v, col0);
  const LiveCols lv{v.live};
  if (v.K > 0)
    x3_gemm<3, 15, 2>(name, zero_net(v), w, h, X3Vocab<LOSS, true>{e}, cols, v.rows, v.H, v.H, s, lv);
  else
    x3_gemm<3, 15, 2>(name, zero_net(v), w, h, X3Vocab<LOSS, false>{e}, cols, v.rows, v.H, v.H, s, lv);
}
template <bool LOSS>
void logits(const char* name, const VocabNet& v, int col0, int cols, hipStream_t s) {
  if (v.C % 4 == 0) logits<LOSS, X3Whole<X3Cols>>(name, v, col0, cols, s);
  else logits<LOSS, X3WCols>(name, v, col0, cols, s);
}

// The loss of few rows or words: 128 words x 64 rows to a workgroup, four
// wavefronts of 32 x 64, two stages of 32 k in flight in registers, split on
// their way to LDS (split3.h's parts, a plane of 64-byte rows each).  W_s is read
// as it is, at the alignment of its elements.  FB: groups of 16 rows; of at most 16
// one alone (4 x 50 001 x 1024: 51 us, 67 with all four).  The 128 x 128 tiles, one chunk in
// flight and twice the work, took 83 us for 9 rows, 8 043 words, H = 1152.
constexpr int kFewWords = 128;
template <bool TEACH, int FB>
__global__ void __launch_bounds__(256, 2) k_vocab_few_x3(VocabEp e, const float* __restrict__ W,
                                                         const float* __restrict__ hp, int H) {
  constexpr int FA = 2, kA = kFewWords * 64, kB = 16 * FB * 64, kPlanes = 3 * (kA + kB);
  __shared__ __attribute__((aligned(16))) char lds[2][kPlanes];
  __shared__ float stats[3][4][kVocabFew];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g = lane >> 4, r = lane & 15;
  const int a0 = blockIdx.x * kFewWords, row0 = blockIdx.y * kVocabFew, C = e.C;
  if (row0 >= *e.live) return;
  const size_t end = (size_t)H * C;   // at least 64 values
  // A: words 2 lane, 2 lane + 1, k octet w; B: row tid / 4, octet tid % 4
  const float* hb = hp + (size_t)(row0 + (tid >> 2)) * H + 8 * (tid & 3);
  struct Stage {
    float2 a[8];
    float4 b[2];
  } st[2];
  auto load = [&](Stage& x, int k0) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const size_t o = (size_t)(k0 + 8 * w + k) * C + a0 + 2 * lane;
      if (o + 2 <= end) __builtin_memcpy(&x.a[k], W + o, 8);
      else x.a[k] = make_float2(o < end ? W[o] : 0.f, 0.f);
    }
    if (FB == 4 || tid < 64 * FB) {
      x.b[0] = ldg4(hb + k0);
      x.b[1] = ldg4(hb + k0 + 4);
    }
  };
  auto put = [&](char* base, int plane, int row, int octet, const float (&v)[8]) {
    const Split8 p = split8(v);
#pragma unroll
    for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4*>(base + k * plane + x3_addr(row, octet)) = p.p[k];
  };
  v4f acc[FA][FB];
  zero_acc(acc);
  load(st[0], 0);
  load(st[1], min(kBK, H - kBK));
  for (int k0 = 0; k0 < H; k0 += 2 * kBK) {   // H is a multiple of 64
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      char* L = lds[s];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = c ? st[s].a[k].y : st[s].a[k].x;
        put(L, kA, 2 * lane + c, w, v);
      }
      if (FB == 4 || tid < 64 * FB) {
        const float4 b0 = st[s].b[0], b1 = st[s].b[1];
        const float v[8] = {b0.x, b0.y, b0.z, b0.w, b1.x, b1.y, b1.z, b1.w};
        put(L + 3 * kA, kB, tid >> 2, tid & 3, v);
      }
      __syncthreads();   // the other buffer's readers are past this one's barrier
      load(st[s], min(k0 + (s + 2) * kBK, H - kBK));   // past the end: the last stage, unused
      __builtin_amdgcn_sched_barrier(0);   // the loads go out before these products
      bf16x8 b[3][FB];
#pragma unroll
      for (int p = 0; p < 3; ++p)
#pragma unroll
        for (int f = 0; f < FB; ++f)
          b[p][f] = *reinterpret_cast<const bf16x8*>(L + 3 * kA + p * kB + x3_addr(16 * f + r, g));
#pragma unroll
      for (int i = 0; i < FA; ++i) {
        bf16x8 a[3];
#pragma unroll
        for (int p = 0; p < 3; ++p)
          a[p] = *reinterpret_cast<const bf16x8*>(L + p * kA + x3_addr(32 * w + 16 * i + r, g));
#pragma unroll
        for (int t = 0; t < kSplitTerms; ++t)
#pragma unroll
          for (int f = 0; f < FB; ++f)
            acc[i][f] = mfma_bf16_16x16x32(a[kTermA[t]], b[kTermB[t]][f], acc[i][f]);
      }
    }
  }
  float nan = 0.f;
#pragma unroll
  for (int i = 0; i < FA; ++i)
#pragma unroll
    for (int f = 0; f < FB; ++f)
#pragma unroll
      for (int q = 0; q < 4; ++q) nan += acc[i][f][q];
  if (nan != nan) {   // NaN, or an operand without parts (split3.h): these words' sums in fp32
#pragma unroll
    for (int i = 0; i < FA; ++i)
#pragma unroll
      for (int f = 0; f < FB; ++f)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int c = a0 + 32 * w + 16 * i + 4 * g + q;
          float s = 0.f;
          if (c < C)
            for (int k = 0; k < H; ++k) s = fmaf(W[(size_t)k * C + c], hp[(size_t)(row0 + 16 * f + r) * H + k], s);
          acc[i][f][q] = s;
        }
  }
  vocab_few_end<TEACH, 64, FB>(e, stats, a0, row0, [&](int i, int f) { return acc[i >> 2][f][i & 3]; });
}

}  // namespace

void vocab_x3_loss(const VocabNet& v, const void* W, hipStream_t s) {
  if (v.small) {
    const dim3 grid(cdiv(v.C, kFewWords), cdiv(v.n, kVocabFew));
    const VocabEp e = vocab_ep(v, 0);
    auto go = [&](auto* kernel) {
      CAVS_LAUNCH("k_vocab_few_x3", kernel, grid, dim3(256), 0, s, e, (const float*)W, (const float*)v.hp, v.H);
    };
    if (v.n <= 16) v.K > 0 ? go(k_vocab_few_x3<true, 1>) : go(k_vocab_few_x3<false, 1>);
    else v.K > 0 ? go(k_vocab_few_x3<true, 4>) : go(k_vocab_few_x3<false, 4>);
    return;
  }
  vocab_launches(v, [&](int col0, int cols) { logits<true>("k_x3_gemm<vocab loss>", v, col0, cols, s); });
}

void vocab_x3_dz(const VocabNet& v, int col0, int cols, hipStream_t s) {
  logits<false>("k_x3_gemm<vocab dz>", v, col0, cols, s);
}

template <class W>
static void grads(const VocabNet& v, int col0, int cols, const VocabOut& o, hipStream_t s) {
  const int hchunk = cdiv(cdiv(cols, kBK), v.Sh) * kBK;
  const VocabOut sums{v.hpart, v.H, (size_t)v.rows * v.H, v.rows, v.H, 0, col0 > 0, nullptr};
  const X3Product dh(X3Rows{(const float*)v.dZ, v.P, v.rows}, W{{(const float*)v.Ws + col0, v.ldw, v.H}},
                     X3VocabOut{sums}, LiveRows{v.live, cdiv(cols, hchunk)}, v.rows, v.H, cols, hchunk);
  const int nch = cdiv(v.n, kBK), wchunk = cdiv(nch, v.Sw) * kBK;
  const X3Product dw(X3Cols{(const float*)v.hp, v.H, v.H}, X3Cols{(const float*)v.dZ, v.P, v.P}, X3VocabOut{o},
                     LiveK{v.live}, v.H, cols, nch * kBK, wchunk);
  if (wchunk >= hchunk) x3_two("k_x3_two<vocab dw, dh>", zero_net(v), dw, dh, s);   // longer items first
  else x3_two("k_x3_two<vocab dw, dh>", zero_net(v), dh, dw, s);
}

void vocab_x3_grads(const VocabNet& v, int col0, int cols, const VocabOut& o, hipStream_t s) {
  if (v.C % 4 == 0) grads<X3Whole<X3Rows>>(v, col0, cols, o, s);
  else grads<X3WRows>(v, col0, cols, o, s);
}

}  // namespace cavs
