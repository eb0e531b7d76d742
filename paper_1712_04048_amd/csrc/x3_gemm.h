// Products on the bf16 matrix cores with operands split (fp32) or rounded
// (bf16) on their way to LDS (split3.h): the operand loaders, the 128 x 128
// tile kernel and its launcher.  A product is built from a loader for each
// side and from what a workgroup does with its tile.
#pragma once

#include <type_traits>

#include "kernels.h"
#include "split3.h"
#include "xcd_map.h"

namespace cavs {

// Operand loaders: thread t of 128 fetches 32 values of the 128-row, 32-deep
// chunk at k0 (zeros past the operand or past kend) and writes them, split,
// to LDS rows 32 j + i (tile rows 4 i + j).
//
// Rows contiguous in k: four adjacent rows, eight k each.
struct X3Rows {
  const float* base;
  long long ld;
  int rows;
  struct State {
    const float* p[4];
    int q, i;
  };
  __device__ void init(const Net&, State& s, int t, int r0) const {
    s.q = t & 3;
    s.i = t >> 2;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = r0 + 4 * s.i + j;
      s.p[j] = r < rows ? base + (size_t)r * ld + 8 * s.q : nullptr;
    }
  }
  __device__ void load(const Net& n, const State& s, int k0, int kend, float4 (&v)[8]) const {
    const int k = k0 + 8 * s.q;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int h = 0; h < 2; ++h)   // K is a multiple of 4
        v[2 * j + h] = ldg4(s.p[j] && k + 4 * h < kend ? s.p[j] + k0 + 4 * h : n.zrow);
  }
  template <int PARTS>
  __device__ static void store(char* lds, const State& s, const float4 (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float x[8] = {v[2 * j].x,     v[2 * j].y,     v[2 * j].z,     v[2 * j].w,
                          v[2 * j + 1].x, v[2 * j + 1].y, v[2 * j + 1].z, v[2 * j + 1].w};
      x3_store<PARTS>(lds, 32 * j + s.i, s.q, x);
    }
  }
};

// k-major: eight k rows, four adjacent columns.
struct X3Cols {
  const float* base;
  long long ld;
  int cols;
  struct State {
    const float* p;
    long long ld;
    int q, i;
  };
  __device__ void init(const Net&, State& s, int t, int r0) const {
    s.q = t >> 5;
    s.i = t & 31;
    const int c = r0 + 4 * s.i;
    s.ld = ld;
    s.p = c < cols ? base + c : nullptr;
  }
  __device__ void load(const Net& n, const State& s, int k0, int kend, float4 (&v)[8]) const {
    const int k = k0 + 8 * s.q;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = ldg4(s.p && k + e < kend ? s.p + (k + e) * s.ld : n.zrow);
  }
  template <int PARTS>
  __device__ static void store(char* lds, const State& s, const float4 (&v)[8]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = j == 0 ? v[e].x : j == 1 ? v[e].y : j == 2 ? v[e].z : v[e].w;
      x3_store<PARTS>(lds, 32 * j + s.i, s.q, x);
    }
  }
};

// What a workgroup does with its 128 x 128 block: lane (r, g) of wavefront
// (wm, wn) holds rows 64 wm + 16 g + 4 e + j, columns 64 wn + 4 r .. + 3.
// Plain: out[z][m][c] (one block per split z of the contraction).
struct X3Out {
  float* out;
  long long ld;
  int rows, cols;
  __device__ void operator()(const Net&, int z, int m0, int n0, int wm, int wn, int g, int r,
                             const v4f (&acc)[4][4]) const {
    float* o = out + (size_t)z * rows * cols;
    const int nc = n0 + 64 * wn + 4 * r;
    if (nc >= cols) return;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int m = m0 + 64 * wm + 16 * g + 4 * e + j;
        if (m < rows)
          st4(o + (size_t)m * ld + nc,
              make_float4(acc[j][0][e], acc[j][1][e], acc[j][2][e], acc[j][3][e]));
      }
  }
};

// The sum over k in [z kchunk, (z + 1) kchunk) of A B^T into ep; the tile and
// its pipeline as in k_x3_tn (lazy.hip).  PARTS: 3 (split fp32) or 1 (bf16).
// Items: bands of kX3Band column tiles, a band's row tiles one after the other,
// a contiguous eighth to each XCD: the 96 tiles that an XCD has in flight are
// then about 8 x 12 and share their operands' rows in its L2.  WGS workgroups
// share a CU.  LV: the product's size where only the device knows it (X3Sized:
// it is the launch's).
struct X3Sized {
  __device__ void operator()(int&, int&, int&, int&) const {}
};
constexpr int kX3Band = 8;
template <int PARTS, int BLOCKS, class LA, class LB, class EP>
__device__ __forceinline__ void x3_tile(char* lds, const Net& n, const LA& la, const LB& lb, const EP& ep,
                                        int ty, int tx, int K, int kchunk, int item) {
  constexpr int OPB = PARTS * kX3Plane;
  const int tid = threadIdx.x, w = tid >> 6, lane = tid & 63, g = lane >> 4, r = lane & 15;
  const int wm = w & 1, wn = w >> 1, z = item / (tx * ty), it = item % (tx * ty);
  const int band = it / (kX3Band * ty), in = it % (kX3Band * ty);
  const int bw = min(kX3Band, tx - band * kX3Band);
  const int m0 = in / bw * kX3Tile, n0 = (band * kX3Band + in % bw) * kX3Tile;
  const int klo = z * kchunk, khi = min(K, klo + kchunk);
  const bool bside = __builtin_amdgcn_readfirstlane(tid >> 7) != 0;
  v4f acc[4][4];
  auto sum = [&](auto parts, int t, auto&& mma) {
    constexpr int P = decltype(parts)::value;
    typename LA::State sa{};
    typename LB::State sb{};
    if (bside) lb.init(n, sb, t, n0);
    else la.init(n, sa, t, m0);
    float4 v[8];
    auto load = [&](int k0) {
      if (bside) lb.load(n, sb, k0, khi, v);
      else la.load(n, sa, k0, khi, v);
    };
    zero_acc(acc);
    if (klo < khi) load(klo);
    for (int k0 = klo; k0 < khi; k0 += kBK) {
      if (k0 > klo) __syncthreads();   // the previous chunk's fragments are read
      if (bside) LB::template store<P>(lds + OPB, sb, v);
      else LA::template store<P>(lds, sa, v);
      __syncthreads();
      if (k0 + kBK < khi) load(k0 + kBK);
      __builtin_amdgcn_sched_barrier(0);   // the next chunk's loads go out before these products
      mma();
    }
  };
  sum(std::integral_constant<int, PARTS>{}, tid & 127,
      [&] { x3_mma<PARTS, BLOCKS>(lds, lds + OPB, wm, wn, acc); });
  if constexpr (PARTS == 3)
    if (x3_nan(acc))   // NaN, or an operand without parts (split3.h)
      sum(std::integral_constant<int, 0>{}, x3_again(tid & 127),
          [&] { x3_mma_f32(lds, lds + OPB, wm, wn, acc); });
  ep(n, z, m0, n0, wm, wn, g, r, acc);
}

template <class LA, class LB, class EP, class LV, int PARTS, int BLOCKS, int WGS>
__global__ void __launch_bounds__(256, WGS) k_x3_gemm(Net n, LA la, LB lb, EP ep, LV lv, int ty,
                                                      int tx, int K, int kchunk, int items) {
  __shared__ __attribute__((aligned(16))) char lds[2 * PARTS * kX3Plane];
  lv(ty, tx, K, items);
  const int item = xcd_item(blockIdx.x, items);
  if (item < 0) return;
  x3_tile<PARTS, BLOCKS>(lds, n, la, lb, ep, ty, tx, K, kchunk, item);
}

template <int PARTS, int BLOCKS, int WGS, class LA, class LB, class EP, class LV = X3Sized>
void x3_gemm(const char* name, const Net& n, LA la, LB lb, EP ep, int M, int Nc, int K, int kchunk,
             hipStream_t s, LV lv = LV{}) {
  const int ty = cdiv(M, kX3Tile), tx = cdiv(Nc, kX3Tile);
  const int items = tx * ty * (K > 0 ? cdiv(K, kchunk) : 1);
  CAVS_LAUNCH(name, (k_x3_gemm<LA, LB, EP, LV, PARTS, BLOCKS, WGS>), dim3(xcd_grid(items)), dim3(256),
              0, s, n, la, lb, ep, lv, ty, tx, K, kchunk, items);
}

// Two independent products of split operands in one launch, the first one's
// workgroups first: either fills the CUs that the other leaves.
template <class LA, class LB, class EP, class LV>
struct X3Product {
  LA la;
  LB lb;
  EP ep;
  LV lv;
  int ty, tx, K, kchunk, items;
  X3Product(LA a, LB b, EP e, LV l, int M, int Nc, int K_, int kchunk_)
      : la(a), lb(b), ep(e), lv(l), ty(cdiv(M, kX3Tile)), tx(cdiv(Nc, kX3Tile)), K(K_), kchunk(kchunk_),
        items(ty * tx * cdiv(K_, kchunk_)) {}
};
template <class P, class Q>
__global__ void __launch_bounds__(256, 2) k_x3_two(Net n, P p, Q q) {
  __shared__ __attribute__((aligned(16))) char lds[2 * 3 * kX3Plane];
  p.lv(p.ty, p.tx, p.K, p.items);
  q.lv(q.ty, q.tx, q.K, q.items);
  const int x = blockIdx.x & 7, at = blockIdx.x >> 3, per = (p.items + 7) / 8;
  if (at < per) {
    const int item = x * per + at;
    if (item < p.items) x3_tile<3, 15>(lds, n, p.la, p.lb, p.ep, p.ty, p.tx, p.K, p.kchunk, item);
  } else {
    const int per2 = (q.items + 7) / 8, item = x * per2 + at - per;
    if (at - per < per2 && item < q.items)
      x3_tile<3, 15>(lds, n, q.la, q.lb, q.ep, q.ty, q.tx, q.K, q.kchunk, item);
  }
}
template <class P, class Q>
void x3_two(const char* name, const Net& n, const P& p, const Q& q, hipStream_t s) {
  CAVS_LAUNCH(name, (k_x3_two<P, Q>), dim3(xcd_grid(p.items) + xcd_grid(q.items)), dim3(256), 0, s, n, p, q);
}

}  // namespace cavs
