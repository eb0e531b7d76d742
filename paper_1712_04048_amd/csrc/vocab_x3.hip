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

// Words are the tile's rows: lane (r, g) holds words 64 wm + 16 g + 4 e + j of
// rows 64 wn + 4 r + c.
template <bool LOSS, bool TEACH>
struct X3Vocab {
  using UsesLds = void;
  VocabEp e;
  __device__ void operator()(char* lds, int, int m0, int n0, int wm, int wn, int g, int r,
                             const v4f (&acc)[4][4]) const {
    const int w = threadIdx.x >> 6, a0 = e.col0 + m0 + 64 * wm, row0 = n0 + 64 * wn;
    auto col = [](int i, int gg) { return 16 * gg + i; };
    float b[16], db[1] = {0.f};
    vocab_bias(e, a0, g, col, b);
    if (!LOSS || TEACH) __syncthreads();   // the slabs take the operands' place
    float* slab = reinterpret_cast<float*>(lds) + w * kSlabFloats<64>;
    const int live = *e.live;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      float z[16];
#pragma unroll
      for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int j = 0; j < 4; ++j) z[4 * q + j] = acc[j][c][q] + b[4 * q + j];
      vocab_rows16<LOSS, TEACH, float, 64>(e, z, col, row0 + c, 4, a0, a0 / 64, live, slab, db);
    }
    if (!LOSS) e.dbp[(size_t)(row0 / 64) * e.ldz + (a0 - e.col0) + (threadIdx.x & 63)] = db[0];
  }
};
static_assert(4 * kSlabFloats<64> * sizeof(float) <= 2 * kX3Bytes, "slabs fit the operands' LDS");

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

template <bool LOSS>
void logits(const char* name, const VocabNet& v, int col0, int cols, hipStream_t s) {
  const X3Cols w{(const float*)v.Ws + col0, v.ldw, std::min(cols, v.Cq - col0)};
  const X3Rows h{(const float*)v.hp, v.H, v.rows};
  const VocabEp e = vocab_ep(v, col0);
  const LiveCols lv{v.live};
  if (v.K > 0)
    x3_gemm<3, 15, 2>(name, zero_net(v), w, h, X3Vocab<LOSS, true>{e}, cols, v.rows, v.H, v.H, s, lv);
  else
    x3_gemm<3, 15, 2>(name, zero_net(v), w, h, X3Vocab<LOSS, false>{e}, cols, v.rows, v.H, v.H, s, lv);
}

}  // namespace

void vocab_x3_loss(const VocabNet& v, hipStream_t s) {
  logits<true>("k_x3_gemm<vocab loss>", v, 0, v.C, s);
}

void vocab_x3_dz(const VocabNet& v, int col0, int cols, hipStream_t s) {
  logits<false>("k_x3_gemm<vocab dz>", v, col0, cols, s);
}

void vocab_x3_dh(const VocabNet& v, int col0, int cols, hipStream_t s) {
  // a quad past C is the padded copy's zeros (X3Rows reads whole quads)
  const int K = cols, kchunk = cdiv(cdiv(K, kBK), v.Sh) * kBK;
  const VocabOut o{v.hpart, v.H, (size_t)v.rows * v.H, v.rows, v.H, 0, col0 > 0, nullptr};
  x3_gemm<3, 15, 2>("k_x3_gemm<vocab dh>", zero_net(v), X3Rows{(const float*)v.dZ, v.P, v.rows},
                    X3Rows{(const float*)v.Ws + col0, v.ldw, v.H}, X3VocabOut{o}, v.rows, v.H, K,
                    kchunk, s, LiveRows{v.live, cdiv(K, kchunk)});
}

void vocab_x3_dw(const VocabNet& v, int col0, int cols, const VocabOut& o, hipStream_t s) {
  const int nch = cdiv(v.rows, kBK), kchunk = cdiv(nch, v.Sw) * kBK;
  x3_gemm<3, 15, 2>("k_x3_gemm<vocab dw>", zero_net(v), X3Cols{(const float*)v.hp, v.H, v.H},
                    X3Cols{(const float*)v.dZ, v.P, v.P}, X3VocabOut{o}, v.H, cols, v.rows,
                    kchunk, s, LiveK{v.live});
}

}  // namespace cavs
