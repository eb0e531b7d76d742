// The vocabulary head outside the cells: softmax cross entropy and distillation
// over z = h W_s + b_s without keeping z.  Shared by its row kernels
// (vocab.hip), its fp32 products (vocab_x3.hip) and its bf16 ones
// (vocab_bf.hip).
//
// Rows without a label take no part: the live rows are listed first (rows[],
// ascending) and everything below works on that compact numbering, whose
// length only the device knows (live[0]).  Every buffer by row has kVocabRows-
// padded capacity; rows from the live ones to the end of their tile hold zeros.
#pragma once

#include "kernels.h"

namespace cavs {

constexpr int kVocabTile = 256;   // rows, and words of a piece, are padded to this
constexpr int kVocabMaxK = 256;   // most teacher's words per row

struct VocabNet {
  int n, H, C, K;
  int rows;                // n padded to kVocabTile
  int bf;                  // products in bf16 (h and W_s rounded), else split fp32
  int hbf, wbf;            // element types of h / dh and of W_s / dW_s
  int two;                 // a second softmax, at a temperature other than 1
  float alpha, temp;
  // dz is kept in units of `unit` = 1 - alpha (alpha = 1: T), so that the label's
  // share is 1 - p and the rounding to bf16 of the rows' common factor (1 / rows,
  // the weights) is not in it: that factor alone, rounded, put dW_s of cross
  // entropy over 7168 rows 0.34 % off instead of 0.18 %.  scal joins the sums.
  float unit, distw;       // distw: alpha T in that unit
  const void* h;
  const void* Ws;          // [H, ldw] of the products' type: the caller's, or its padded copy
  long long ldw;
  int Cq;                  // readable columns of Ws (a multiple of 16 bytes)
  const float* bs;
  // workspace
  int* rows_list;          // [rows] live row -> caller's row
  int* place;              // [n] caller's row -> live row, or -1
  int* live;               // [0] live rows
  float* scal;             // [0] unit / max(1, live rows)
  int* label;              // [rows] -1: none
  int* tword;              // [rows, K] distinct words of the row, -1: none
  float* tq;               // [rows, K] the teacher's probability of tword
  float2* tsum;            // [rows] sum of q ln q, 1 (a teacher's word is there) or 0
  void* hp;                // [rows, H] live rows of h in the products' type
  float* pm;               // [slots, rows] each slot of columns: its largest z,
  float* ps;               //   sum of exp(z - largest),
  float* pt;               //   and of exp((z - largest) / temp) (two)
  int slots, slot_words;   // words of a slot
  float* zlab;             // [rows] z of the label
  float* ztop;             // [rows, K] z of tword
  float4* rowc;            // [rows] largest z, weight of exp(z - largest), weight of
                           //   exp((z - largest) / temp), weight of the label
  float* val;              // [rows] the row's loss
  float* zrow;             // a row of zeros (16 bytes and more)
  // gradient, one piece of words at a time
  int P;                   // words of a piece, a multiple of kVocabTile
  void* dZ;                // [rows, P] products' type
  float* dbp;              // [rows / 64 or finer, P] sums of dz over groups of rows
  int db_rows;             // rows of a group
  float* hpart;            // [Sh, rows, H] dh's sums, added to by each piece
  int Sh;
  float* wpart;            // [Sw, H, P]: dW's sums of a piece (Sw > 1)
  int Sw;
};

// What the products' epilogues read and write.
struct VocabEp {
  int C, col0, K, rows, two;
  float invT, distw;
  const int* live;
  const float* bs;
  const int* label;
  const int* tword;
  const float* tq;
  float *pm, *ps, *pt, *zlab, *ztop;
  const float4* rowc;
  void* dz;
  long long ldz;
  float* dbp;
};

// Where dh's and dW's sums go: rows x cols of out (+ z * part), added to what
// is there or not, times *scale (null: 1), stored as float or bf16.
struct VocabOut {
  void* out;
  long long ld;
  size_t part;
  int rows, cols, bf, acc;
  const float* scale;
};

__device__ __forceinline__ void wave_lds_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// LDS floats of a wavefront's slab: 16 rows of NC columns, four floats of
// padding (a lane group's 16-byte writes to 16 rows then spread over the banks).
template <int NC>
constexpr int kSlabFloats = 16 * (NC + 4);

// One group of 16 rows of a wavefront's tile: lane (g, r) holds NV = NC / 4 of
// row `row` (its own r's; rr's row is row0 + step rr), z[i] the product of word
// a0 + col(i, g).  LOSS: the slot's statistics and the z that the loss names.
// Otherwise dz = w1 exp(z - m) + wT exp((z - m) / T) - [label] - teacher's q,
// in 32 bits until it is stored, and its sum over the rows into db.
//
// The statistics need one pass: largest, then the sums relative to it, which
// the row kernel joins over the slots.  A slot without a finite word (words
// masked with -inf, columns past C) has largest -inf and sums 0.
template <bool LOSS, bool TEACH, class OUT, int NC, class Col>
__device__ __forceinline__ void vocab_rows16(const VocabEp& e, float (&z)[NC / 4], Col col, int row0,
                                             int step, int a0, int slot, int live, float* slab,
                                             float (&db)[NC / 64]) {
  constexpr int NV = NC / 4, LD = NC + 4;
  const int lane = threadIdx.x & 63, g = lane >> 4, r = lane & 15, row = row0 + step * r;
  const bool here = row < live;
  const int lab = here && e.label ? e.label[row] - a0 : -1;
  if constexpr (LOSS) {
    float m = z[0];
#pragma unroll
    for (int i = 1; i < NV; ++i) m = fmaxf(m, z[i]);
    m = fmaxf(m, __shfl_xor(m, 16, kWave));
    m = fmaxf(m, __shfl_xor(m, 32, kWave));
    const float mm = m == -INFINITY ? 0.f : m;
    float s = 0.f, t = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) s += __builtin_amdgcn_exp2f((z[i] - mm) * kLog2e);
    s += __shfl_xor(s, 16, kWave);
    s += __shfl_xor(s, 32, kWave);
    if (e.two) {
#pragma unroll
      for (int i = 0; i < NV; ++i) t += __builtin_amdgcn_exp2f((z[i] - mm) * e.invT * kLog2e);
      t += __shfl_xor(t, 16, kWave);
      t += __shfl_xor(t, 32, kWave);
    }
    if (g == 0) {
      const size_t at = (size_t)slot * e.rows + row;
      e.pm[at] = m;
      e.ps[at] = s;
      if (e.two) e.pt[at] = t;
    }
    if ((unsigned)lab < (unsigned)NC) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (col(i, g) == lab) e.zlab[row] = z[i];
    }
  } else {
    float4 c = e.rowc[row];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float v = c.y * __builtin_amdgcn_exp2f((z[i] - c.x) * kLog2e);
      if (e.two) v += c.z * __builtin_amdgcn_exp2f((z[i] - c.x) * e.invT * kLog2e);
      if (col(i, g) == lab) v -= c.w;
      z[i] = here && a0 + col(i, g) < e.C ? v : 0.f;
    }
  }
  if constexpr (!LOSS || TEACH) {
    // four adjacent words of a lane at a time
#pragma unroll
    for (int i = 0; i < NV; i += 4)
      st4(slab + r * LD + col(i, g), make_float4(z[i], z[i + 1], z[i + 2], z[i + 3]));
    wave_lds_fence();
  }
  if constexpr (TEACH) {
    // each teacher's word of a row is there once (k_vocab_teacher), so no two
    // lanes change one place
    for (int x = lane; x < 16 * e.K; x += 64) {
      const int rr = (unsigned)x / (unsigned)e.K, rw = row0 + step * rr;
      if (rw >= live) continue;
      const size_t at = (size_t)rw * e.K + (x - rr * e.K);
      const int d = e.tword[at] - a0;
      if ((unsigned)d >= (unsigned)NC) continue;
      if constexpr (LOSS) e.ztop[at] = slab[rr * LD + d];
      else slab[rr * LD + d] -= e.distw * e.tq[at];
    }
    wave_lds_fence();
  }
  if constexpr (!LOSS) {
#pragma unroll
    for (int k = 0; k < NC / 64; ++k)
#pragma unroll
      for (int rr = 0; rr < 16; ++rr) db[k] += slab[rr * LD + lane + 64 * k];
    constexpr int VEC = sizeof(OUT) == 2 ? 8 : 4, PER = NC / VEC, ROWS = 64 / PER;
    const int rr0 = lane / PER, c0 = lane % PER * VEC;
#pragma unroll
    for (int k = 0; k < 16 / ROWS; ++k) {
      const int rr = rr0 + k * ROWS;
      OUT* d = (OUT*)e.dz + (size_t)(row0 + step * rr) * e.ldz + (a0 - e.col0) + c0;
      const float4 x = *reinterpret_cast<const float4*>(slab + rr * LD + c0);
      if constexpr (sizeof(OUT) == 2) {
        const float4 y = *reinterpret_cast<const float4*>(slab + rr * LD + c0 + 4);
        *reinterpret_cast<uint4*>(d) =
            make_uint4(f2bf2(x.x, x.y), f2bf2(x.z, x.w), f2bf2(y.x, y.y), f2bf2(y.z, y.w));
      } else {
        *reinterpret_cast<float4*>(d) = x;
      }
    }
    wave_lds_fence();   // the next group's values overwrite the slab
  } else if constexpr (TEACH) {
    wave_lds_fence();
  }
}

// The bias of a lane's words (0 where there is none), for words past C -inf:
// added to the product, it takes them out of the softmax.
template <int NV, class Col>
__device__ __forceinline__ void vocab_bias(const VocabEp& e, int a0, int g, Col col, float (&b)[NV]) {
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = a0 + col(i, g);
    b[i] = c < e.C ? (e.bs ? e.bs[c] : 0.f) : -INFINITY;
  }
}

// four adjacent values of one row of an output, times w
__device__ __forceinline__ void vocab_store4(const VocabOut& o, float w, int z, int row, int c, float4 v) {
  if (row >= o.rows || c >= o.cols) return;
  v = make_float4(v.x * w, v.y * w, v.z * w, v.w * w);
  const size_t at = z * o.part + (size_t)row * o.ld + c;
  const float x[4] = {v.x, v.y, v.z, v.w};
  if (o.bf) {
    u16* d = (u16*)o.out + at;
    if ((o.ld & 3) == 0 && c + 4 <= o.cols) {
      st_bf4(d, v);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (c + i < o.cols) d[i] = f2bf(x[i]);
    }
  } else {
    float* d = (float*)o.out + at;
    if ((o.ld & 3) == 0 && c + 4 <= o.cols) {
      st4(d, o.acc ? add4(ldg4(d), v) : v);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (c + i < o.cols) d[i] = o.acc ? d[i] + x[i] : x[i];
    }
  }
}

VocabEp vocab_ep(const VocabNet& v, int col0);

// The products, by type.  loss: statistics of every word; dz: one piece's dZ
// and dbp; dh: the piece's share of hpart; dW: the piece's columns of dW.
void vocab_x3_loss(const VocabNet& v, hipStream_t s);
void vocab_x3_dz(const VocabNet& v, int col0, int cols, hipStream_t s);
void vocab_x3_dh(const VocabNet& v, int col0, int cols, hipStream_t s);
void vocab_x3_dw(const VocabNet& v, int col0, int cols, const VocabOut& o, hipStream_t s);
void vocab_bf_loss(const VocabNet& v, hipStream_t s);
void vocab_bf_dz(const VocabNet& v, int col0, int cols, hipStream_t s);
void vocab_bf_dh(const VocabNet& v, int col0, int cols, hipStream_t s);
void vocab_bf_dw(const VocabNet& v, int col0, int cols, const VocabOut& o, hipStream_t s);

// embed.hip
size_t embed_grad_ws_bytes(const cavs_embedding* e, int n);
cavs_status embed_run(cavs_ctx* ctx, const cavs_embedding* e, const int* word, int n, void* X);
cavs_status embed_grad_run(cavs_ctx* ctx, const cavs_embedding* e, const int* word, int n,
                           const void* dX, void* dE, void* ws, size_t ws_bytes);

// vocab.hip
size_t vocab_ws_bytes(const cavs_vocab* p, bool train);
cavs_status vocab_run(cavs_ctx* ctx, const cavs_vocab* p, float* loss, float* row_loss, void* dh,
                      void* dWs, float* dbs, void* ws, size_t ws_bytes, bool train);

}  // namespace cavs
