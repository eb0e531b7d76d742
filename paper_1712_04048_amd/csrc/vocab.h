// The vocabulary head outside the cells: softmax cross entropy and distillation
// over z = h W_s + b_s without keeping z.  Shared by its row kernels
// (vocab.hip), its fp32 products (vocab_x3.hip) and its bf16 ones
// (vocab_bf.hip).
//
// Rows without a label take no part: the live rows are listed first (rows[],
// ascending) and everything below works on that compact numbering, whose
// length only the device knows (live[0]).  Every buffer by row has a capacity of
// n padded to kVocabTile, or kVocabFew of at most that many: those take no tile of
// 256 rows but of operands whose rows it bounds, and keep z, so that no such tile
// forms their dz.  The rows of hp and dZ that follow the live ones in the gradients'
// contraction hold zeros.
#pragma once

#include <algorithm>
#include <type_traits>

#include "kernels.h"

namespace cavs {

constexpr int kVocabTile = 256;   // rows, and words of a piece, are padded to this
constexpr int kVocabFew = 64;     // most rows of the kernels for few rows
constexpr int kVocabMaxK = 256;   // most teacher's words per row

struct VocabNet {
  int n, H, C, K;
  int rows;                // n padded to kVocabTile (few: to kVocabFew)
  int bf;                  // products in bf16 (h and W_s rounded), else split fp32
  int hbf, wbf;            // element types of h / dh and of W_s / dW_s
  int few, pad, keep;      // at most kVocabFew rows; Ws is a padded copy; z is kept
  int small;               // the loss on tiles of 128 words x 64 rows
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
  int Cq;                  // bf16: readable columns of Ws (a multiple of 16 bytes)
  const float* bs;
  // workspace
  int* rows_list;          // [rows] live row -> caller's row
  int* place;              // [n] caller's row -> live row, or -1
  int* live;               // [0] live rows
  float* scal;             // [0] unit / max(1, live rows)
  int* label;              // [rows] -1: none
  int* tword;              // [rows, K] the row's words, ascending (absent ones last)
  float* tq;               // [rows, K] the teacher's probability of tword (a word that
                           //   is there twice: all of it at its first place, else 0)
  uint32_t* trange;        // [slots, rows] places in tword of the words of a slot: the
                           //   first, and past the last in the upper half
  float2* tsum;            // [rows] sum of q ln q, 1 (a teacher's word is there) or 0
  void* hp;                // [rows, H] live rows of h in the products' type
  float* pm;               // [slots, rows] each slot of columns: its largest z,
  float* ps;               //   sum of exp(z - largest),
  float* pt;               //   and of exp((z - largest) / temp) (two)
  int slots, slot_words;   // words of a slot
  float* zlab;             // [rows] z of the label
  float* ztop;             // [rows, K] z of tword
  float4* rowc;            // [rows] largest z, weight of exp(z - largest), weight of
                           //   exp((z - largest) / temp), weight of the label; inf and
                           //   zeros for a row without dz
  float* val;              // [rows] the row's loss
  float* zrow;             // a row of zeros (16 bytes and more)
  // gradient, one piece of words at a time
  int P;                   // words of a piece, a multiple of kVocabTile
  void* dZ;                // [rows, P] products' type (bf16, several pieces: two of them)
  size_t dz_half;          // bytes from one to the other
  float* Z;                // [rows, P] z in one piece, where it is kept (in fp32 dZ itself), or null
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
  const uint32_t* trange;
  float *pm, *ps, *pt, *zlab, *ztop;
  float* zkeep;            // LOSS: z goes here (or null), rows of ldz
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

// V adjacent elements as they are in memory, as floats, and back (rounded once)
template <int V, class T>
struct RawRow {
  static constexpr int kBytes = V * (int)sizeof(T);
  uint32_t w[(kBytes + 3) / 4];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (kBytes % 16 == 0) {
#pragma unroll
      for (int i = 0; i < kBytes / 16; ++i) {
        const uint4 x = reinterpret_cast<const uint4*>(p)[i];
        w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
      }
    } else if constexpr (kBytes == 8) {
      const uint2 x = *reinterpret_cast<const uint2*>(p);
      w[0] = x.x; w[1] = x.y;
    } else {
      static_assert(V == 1, "16 or 8 bytes, or one element");
      if constexpr (sizeof(T) == 4) w[0] = __float_as_uint(*p);
      else w[0] = *p;
    }
  }
  __device__ __forceinline__ void floats(float (&v)[V]) const {
#pragma unroll
    for (int i = 0; i < V; ++i)
      v[i] = __uint_as_float(sizeof(T) == 4 ? w[i] : i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
  }
};
template <int V, class T>
__device__ __forceinline__ void load_row(const T* p, float (&v)[V]) {
  RawRow<V, T> x;
  x.load(p);
  x.floats(v);
}
template <int V, class T>
__device__ __forceinline__ void store_row(T* p, const float (&v)[V]) {
  if constexpr (sizeof(T) == 4) {
    if constexpr (V % 4 == 0) {
#pragma unroll
      for (int i = 0; i < V; i += 4) st4((float*)p + i, make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]));
    } else {
#pragma unroll
      for (int i = 0; i < V; ++i) p[i] = v[i];
    }
  } else if constexpr (V == 8) {
    *reinterpret_cast<uint4*>(p) =
        make_uint4(f2bf2(v[0], v[1]), f2bf2(v[2], v[3]), f2bf2(v[4], v[5]), f2bf2(v[6], v[7]));
  } else if constexpr (V == 4) {
    st_bf4((u16*)p, make_float4(v[0], v[1], v[2], v[3]));
  } else {
#pragma unroll
    for (int i = 0; i < V; ++i) p[i] = f2bf(v[i]);
  }
}

// The sum over the sixteen lanes of a lane group, in every one of them.
__device__ __forceinline__ float row16_sum(float v) {
  auto ror = [](float x, auto n) {   // row_ror
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), 0x120 + decltype(n)::value, 15, 15, true));
  };
  v += ror(v, std::integral_constant<int, 8>{});
  v += ror(v, std::integral_constant<int, 4>{});
  v += ror(v, std::integral_constant<int, 2>{});
  v += ror(v, std::integral_constant<int, 1>{});
  return v;
}

// What an epilogue needs of a row: its constants (rowc), its label (-1: none, or
// no live row), its teacher's words in the slot.
struct VocabRow {
  float4 c;
  int label;
  uint32_t range;
};
template <bool LOSS, bool TEACH>
__device__ __forceinline__ VocabRow vocab_row(const VocabEp& e, int row, int slot, int live) {
  VocabRow v{};
  if (!LOSS) v.c = e.rowc[row];
  v.label = row < live && e.label ? e.label[row] : -1;
  if (TEACH) v.range = row < live ? e.trange[(size_t)slot * e.rows + row] : 0u;
  return v;
}

// One group of 16 rows of a wavefront's tile of NC words, which lie in one slot
// of words: lane (g, r) holds NV = NC / 4 of row `row` (r's), z[i] the score of word
// a0 + col(i, g), four adjacent i adjacent words.  LOSS: the words' statistics
// (to pm[stat] and on) and the z that the loss names.  Otherwise dz = w1 exp(z - m) + wT exp((z - m)
// / T) - [label] - teacher's q, in 32 bits until it is stored, and added to db.
//
// The statistics need one pass: largest, then the sums relative to it, which
// the row kernel joins over the slots.  A slot without a finite word (words
// masked with -inf, columns past C) has largest -inf and sums 0.
//
// A row's label and its teacher's words fall into few slots, so what looks for
// them is skipped where no row of the group has one: the labels by comparison,
// the words (sorted by k_vocab_teacher) by their range in this slot.  The
// values go out as the lanes hold them: passing them through LDS for whole
// 128-byte stores made a tile of dz 20 us long, where a tile's product of
// depth 1024 is 25.
template <bool LOSS, bool TEACH, class OUT, int NC, class Col>
__device__ __forceinline__ void vocab_rows16(const VocabEp& e, float (&z)[NC / 4], Col col, int row,
                                             const VocabRow& info, int a0, size_t stat,
                                             float (&db)[NC / 4]) {
  constexpr int NV = NC / 4;
  const int g = (threadIdx.x & 63) >> 4;
  const int lab = info.label - a0;   // -1 - a0 is no column either
  const bool labelled = __any((unsigned)lab < (unsigned)NC);
  const uint32_t range = info.range;
  // f(word's place in the row's list, its column) for each of the row's words here
  auto words = [&](auto&& f) {
    const int hi = range >> 16;
    for (int j = range & 0xffffu; __any(j < hi); ++j) {
      const size_t at = (size_t)row * e.K + j;
      f(at, j < hi ? e.tword[at] - a0 : -1);
    }
  };
  if constexpr (LOSS) {
    if (e.zkeep) {
      float* d = e.zkeep + (size_t)row * e.ldz + a0;
#pragma unroll
      for (int i = 0; i < NV; i += 4) st4(d + col(i, g), make_float4(z[i], z[i + 1], z[i + 2], z[i + 3]));
    }
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
    if (TEACH && e.two) {
      const float k = e.invT * kLog2e;
#pragma unroll
      for (int i = 0; i < NV; ++i) t += __builtin_amdgcn_exp2f((z[i] - mm) * k);
      t += __shfl_xor(t, 16, kWave);
      t += __shfl_xor(t, 32, kWave);
    }
    if (g == 0) {
      e.pm[stat] = m;
      e.ps[stat] = s;
      if (TEACH && e.two) e.pt[stat] = t;
    }
    if (labelled) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
        if (col(i, g) == lab) e.zlab[row] = z[i];
    }
    if constexpr (TEACH)
      words([&](size_t at, int d) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (col(i, g) == d) e.ztop[at] = z[i];
      });
  } else {
    const float4 c = info.c;
    // A row in which no exponential counts (behind the last live one, or with the
    // teacher alone and none of its words; c.x is inf) has no dz, whatever its z is:
    // the score of a word that W_s masks with -inf is a NaN where the state is 0, as
    // behind the last row, and would stay one times a weight of 0.
    const bool none = c.y == 0.f && c.z == 0.f;
    if (__any(none)) {
#pragma unroll
      for (int i = 0; i < NV; ++i) z[i] = none ? 0.f : z[i];
    }
    if (TEACH && e.two) {
      const float k = e.invT * kLog2e;
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        const float x = z[i] - c.x;
        z[i] = c.y * __builtin_amdgcn_exp2f(x * kLog2e) + c.z * __builtin_amdgcn_exp2f(x * k);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NV; ++i) z[i] = c.y * __builtin_amdgcn_exp2f((z[i] - c.x) * kLog2e);
    }
    if (labelled) {
#pragma unroll
      for (int i = 0; i < NV; ++i) z[i] -= col(i, g) == lab ? c.w : 0.f;
    }
    if constexpr (TEACH)
      words([&](size_t at, int d) {
        const float q = d >= 0 ? e.distw * e.tq[at] : 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) z[i] -= col(i, g) == d ? q : 0.f;
      });
    if (a0 + NC > e.C) {   // words past C (a row whose sums are NaN has NaN there too)
#pragma unroll
      for (int i = 0; i < NV; ++i) z[i] = a0 + col(i, g) < e.C ? z[i] : 0.f;
    }
    OUT* d = (OUT*)e.dz + (size_t)row * e.ldz + (a0 - e.col0);
#pragma unroll
    for (int i = 0; i < NV; i += 4) {
      const float4 v = make_float4(z[i], z[i + 1], z[i + 2], z[i + 3]);
      if constexpr (sizeof(OUT) == 2) st_bf4((u16*)d + col(i, g), v);
      else st4((float*)d + col(i, g), v);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) db[i] += z[i];
  }
}

// A wavefront's sums of dz over its rows, as group `group` of the piece's.
template <int NC, class Col>
__device__ __forceinline__ void vocab_db(const VocabEp& e, float (&db)[NC / 4], Col col, int a0, int group) {
  const int lane = threadIdx.x & 63, g = lane >> 4;
  float* d = e.dbp + (size_t)group * e.ldz + (a0 - e.col0);
#pragma unroll
  for (int i = 0; i < NC / 4; ++i) db[i] = row16_sum(db[i]);
#pragma unroll
  for (int i = 0; i < NC / 4; i += 4)
    if ((lane & 15) == (i / 4) % 16) st4(d + col(i, g), make_float4(db[i], db[i + 1], db[i + 2], db[i + 3]));
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

// A workgroup of the loss's small tiles: four wavefronts of 32 words each by 16 FB
// rows from row0 on, z(i, f) lane (g, r)'s word col(i, g) of row row0 + 16 f + r.
// The wavefronts' statistics are joined into the slots of SW words.
template <bool TEACH, int SW, int FB, class Z>
__device__ __forceinline__ void vocab_few_end(const VocabEp& e, float (&stats)[3][4][kVocabFew], int a0,
                                              int row0, Z z) {
  constexpr int NC = 32, PER = SW / NC;   // wavefronts of a slot
  const int tid = threadIdx.x, w = tid >> 6, g = (tid & 63) >> 4, r = tid & 15, aw = a0 + NC * w;
  VocabEp own = e;
  own.pm = stats[0][w];
  own.ps = stats[1][w];
  own.pt = stats[2][w];
  auto col = [](int i, int gg) { return 16 * (i >> 2) + 4 * gg + (i & 3); };
  float bias[NC / 4], db[NC / 4];
  vocab_bias(e, aw, g, col, bias);
  const int live = *e.live;
#pragma unroll
  for (int f = 0; f < FB; ++f) {
    float x[NC / 4];
#pragma unroll
    for (int i = 0; i < NC / 4; ++i) x[i] = z(i, f) + bias[i];
    if (aw + NC > e.C) {   // what was read past a row's end is the next row's: any value
#pragma unroll
      for (int i = 0; i < NC / 4; ++i) x[i] = aw + col(i, g) < e.C ? x[i] : -INFINITY;
    }
    const int row = row0 + 16 * f + r;
    vocab_rows16<true, TEACH, float, NC>(own, x, col, row, vocab_row<true, TEACH>(e, row, aw / SW, live), aw,
                                         16 * f + r, db);
  }
  __syncthreads();
  const int row = tid & 63;
  if (w >= 4 / PER || row >= 16 * FB) return;
  float m = -INFINITY, s = 0.f, t = 0.f;
#pragma unroll
  for (int k = 0; k < PER; ++k) m = fmaxf(m, stats[0][PER * w + k][row]);
  const float mm = m == -INFINITY ? 0.f : m;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const float d = (stats[0][PER * w + k][row] - mm) * kLog2e;
    s += stats[1][PER * w + k][row] * __builtin_amdgcn_exp2f(d);
    if (TEACH && e.two) t += stats[2][PER * w + k][row] * __builtin_amdgcn_exp2f(d * e.invT);
  }
  const size_t at = (size_t)(a0 / SW + w) * e.rows + row0 + row;
  e.pm[at] = m;
  e.ps[at] = s;
  if (TEACH && e.two) e.pt[at] = t;
}

// Eight adjacent values from element o on of a matrix of `end` elements (at least
// 64): where it ends among them, or before, what there is and zeros.
__device__ __forceinline__ uint4 vocab_load8(const u16* W, size_t o, size_t end) {
  uint4 x;
  if (o + 8 <= end) {
    __builtin_memcpy(&x, W + o, 16);
  } else {
    unsigned __int128 t;
    __builtin_memcpy(&t, W + (end - 8), 16);
    t = o < end ? t >> (16 * (int)(o - (end - 8))) : 0;
    __builtin_memcpy(&x, &t, 16);
  }
  return x;
}
// The same of one row that has `left` values from o on: zeros behind them.
__device__ __forceinline__ uint4 vocab_row8(const u16* W, size_t o, size_t end, int left) {
  uint4 x = vocab_load8(W, o, end);
  if (left < 8) {
    unsigned __int128 t;
    __builtin_memcpy(&t, &x, 16);
    t = left > 0 ? t & (((unsigned __int128)1 << (16 * left)) - 1) : 0;
    __builtin_memcpy(&x, &t, 16);
  }
  return x;
}

// four adjacent values of one row of an output, times w
__device__ __forceinline__ void vocab_store4(const VocabOut& o, float w, int z, int row, int c, float4 v) {
  if (row >= o.rows || c >= o.cols) return;
  v = make_float4(v.x * w, v.y * w, v.z * w, v.w * w);
  const size_t at = z * o.part + (size_t)row * o.ld + c;
  const float x[4] = {v.x, v.y, v.z, v.w};
  if (o.bf) {
    u16* d = (u16*)o.out + at;
    // at the alignment of an element, whatever C is: dW_s of 50 001 columns and few
    // rows took 106 us in 2-byte stores, 53 so
    if (c + 4 <= o.cols) {
      const uint2 q = make_uint2(f2bf2(v.x, v.y), f2bf2(v.z, v.w));
      __builtin_memcpy(d, &q, 8);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (c + i < o.cols) d[i] = f2bf(x[i]);
    }
  } else {
    float* d = (float*)o.out + at;
    if (c + 4 <= o.cols) {
      if (o.acc) v = add4(ldg4(d), v);   // sums of the library's own, aligned
      __builtin_memcpy(d, &v, 16);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (c + i < o.cols) d[i] = o.acc ? d[i] + x[i] : x[i];
    }
  }
}

VocabEp vocab_ep(const VocabNet& v, int col0);

// f(col0, cols) over the vocabulary, in launches of at most 2^22 tiles: a grid has
// fewer than 2^32 threads.
template <class F>
void vocab_launches(const VocabNet& v, F f) {
  const int step = (int)std::min<size_t>((size_t)1 << 30, ((size_t)1 << 36) / v.rows / kVocabTile * kVocabTile);
  for (int col0 = 0; col0 < v.C; col0 += step) f(col0, std::min(step, v.C - col0));
}

// The piece of dZ that begins with word col0: the two halves in turn.
inline char* vocab_dz_at(const VocabNet& v, int col0) {
  return (char*)v.dZ + (col0 / v.P % 2) * v.dz_half;
}

// The products, by type.  loss: statistics of every word (few rows: from the
// caller's W, without a padded copy); dz: one piece's dZ and dbp; grads:
// the piece's share of hpart (dL/dh) and its columns of dW_s.
void vocab_x3_loss(const VocabNet& v, const void* W, hipStream_t s);
void vocab_x3_dz(const VocabNet& v, int col0, int cols, hipStream_t s);
void vocab_x3_grads(const VocabNet& v, int col0, int cols, const VocabOut& o, hipStream_t s);
void vocab_bf_loss(const VocabNet& v, const void* W, hipStream_t s);
void vocab_bf_dz(const VocabNet& v, int col0, int cols, hipStream_t s);
void vocab_bf_grads(const VocabNet& v, int col0, int cols, int next, const VocabOut& o, hipStream_t s);

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
