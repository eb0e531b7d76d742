// bf16 products of the vocabulary head: operands in bf16 in memory, copied
// straight to LDS (global_load_lds_dwordx4), fp32 accumulation on
// v_mfma_f32_16x16x32_bf16.
#include <algorithm>

#include "lds_ring.h"
#include "vocab.h"
#include "xcd_map.h"

namespace cavs {
namespace {

constexpr int kKB = 64;   // contraction depth of a stage

// An operand's tile of ROWS rows, kKB deep, in LDS, and how it gets there.  A
// workgroup's copy instruction moves 16 bytes per thread, thread t of T to byte
// 16 t, so the swizzles permute what a thread reads, not where it writes.
//
// Contiguous in the contraction: LDS rows of 128 bytes, their eight 16-byte
// quads at quad ^ (row & 7); eight lanes that read one quad of eight rows then
// cover the banks once.  The last quads may lie past the operand's end (kmax):
// they read its last ones instead, which meet zeros of the other operand.
struct RowsOp {
  const u16* p;
  long long ld;
  int rows, kmax;
  template <int ROWS, int T>
  struct Tile {
    static constexpr int kCopies = ROWS * 128 / (16 * T);
    static_assert(kCopies * 16 * T == ROWS * 128, "whole copies");
    const u16* base[kCopies];
    int k, kmax;
    __device__ void init(const RowsOp& o, int r0, int tid) {
      kmax = o.kmax - 8;
#pragma unroll
      for (int i = 0; i < kCopies; ++i) {
        const int at = i * T + tid, row = at >> 3;
        base[i] = o.p + (size_t)min(r0 + row, o.rows - 1) * o.ld;
      }
      k = 8 * ((tid & 7) ^ ((tid >> 3) & 7));   // T is a multiple of 64: the same row & 7 for every i
    }
    __device__ void issue(int k0, uint32_t lds) const {
      const int kk = min(k0 + k, kmax);
#pragma unroll
      for (int i = 0; i < kCopies; ++i)
        copy16_to_lds(reinterpret_cast<const float*>(base[i] + kk), lds + 16 * T * i);
    }
  };
  // rows w0 + 16 f + r, k = 32 kk + 8 g ..
  template <int ROWS>
  struct Frag {
    uint32_t at[2];
    __device__ void init(int w0, int g, int r) {
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) at[kk] = (w0 + r) * 128 + (((4 * kk + g) ^ (r & 7)) << 4);
    }
    __device__ bf16x8 read(const char* lds, int kk, int f) const {
      return *reinterpret_cast<const bf16x8*>(lds + at[kk] + f * 2048);
    }
  };
};

// Contraction-major: LDS rows of ROWS values for each k, their 32-byte segments
// (16 operand rows) at segment ^ s(k), s(k) = (k & 3) | (k >> 3 & 1) << 2.  A
// fragment is two transposing reads (ds_read_b64_tr_b16): sixteen lanes on four
// k and sixteen operand rows get a column of four k each.  The 32 lanes of two
// lane groups read eight k of different s, so their segments cover the banks
// once.
struct ColsOp {
  const u16* p;
  long long ld;
  int cols;   // columns there are (the last eight are read again past them)
  template <int ROWS, int T>
  struct Tile {
    static_assert(ROWS >= 128, "eight segments to permute");
    static constexpr int kCopies = ROWS * 128 / (16 * T);
    static_assert(kCopies * 16 * T == ROWS * 128, "whole copies");
    const u16* base[kCopies];
    long long ld;
    __device__ void init(const ColsOp& o, int c0, int tid) {
      ld = o.ld;
#pragma unroll
      for (int i = 0; i < kCopies; ++i) {
        const int at = i * T + tid, k = at / (ROWS / 8), q = at % (ROWS / 8);
        const int s = (k & 3) | ((k >> 3) & 1) << 2;
        const int c = c0 + 16 * ((q >> 1) ^ s) + 8 * (q & 1);
        base[i] = o.p + (size_t)k * o.ld + min(c, o.cols - 8);
      }
    }
    __device__ void issue(int k0, uint32_t lds) const {
#pragma unroll
      for (int i = 0; i < kCopies; ++i)
        copy16_to_lds(reinterpret_cast<const float*>(base[i] + (size_t)k0 * ld), lds + 16 * T * i);
    }
  };
  template <int ROWS>
  struct Frag {
    int seg0, s;
    uint32_t at;
    __device__ void init(int w0, int g, int r) {
      seg0 = w0 / 16;
      s = (r >> 2) | (g & 1) << 2;
      at = (8 * g + (r >> 2)) * (2 * ROWS) + 8 * (r & 3);
    }
    __device__ bf16x8 read(const char* lds, int kk, int f) const {
      typedef short s4 __attribute__((ext_vector_type(4)));
      typedef short s8 __attribute__((ext_vector_type(8)));
      typedef __attribute__((address_space(3))) s4 lds_s4;
      const char* a = lds + at + (((seg0 + f) ^ s) << 5) + kk * 32 * (2 * ROWS);
      const s4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)a);
      const s4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(a + 4 * (2 * ROWS)));
      const s8 v = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
      return __builtin_bit_cast(bf16x8, v);
    }
  };
};

// How a product's size depends on the live rows: they are its B rows (what 1)
// or its contraction (2).
struct Live {
  const int* live;
  int what;
};

// A workgroup of WA x WB wavefronts: A rows 16 FA WA, B rows 16 FB WB, each
// wavefront 16 FA x 16 FB.  S stages of LDS: a stage's copies are S - 1 stages
// ahead of its products, one barrier a stage.
template <int WA_, int WB_, int FA_, int FB_, int S_>
struct Shape {
  static constexpr int WA = WA_, WB = WB_, FA = FA_, FB = FB_, S = S_;
  static constexpr int T = 64 * WA * WB, BA = 16 * FA * WA, BB = 16 * FB * WB;
  static constexpr int kStage = (BA + BB) * 128, kBytes = S * kStage;
};

constexpr int kBand = 8;
template <class SH, class OA, class OB, class EP>
__global__ void __launch_bounds__(SH::T, 2) k_vocab_bf(OA oa, OB ob, EP ep, Live lv, int ta, int tb,
                                                       int K, int kchunk, int slices) {
  constexpr int FA = SH::FA, FB = SH::FB, S = SH::S;
  __shared__ __attribute__((aligned(16))) char lds[SH::kBytes];
  if (lv.what == 1) tb = cdiv_dev(*lv.live, SH::BB);
  if (lv.what == 2) K = min(K, cdiv_dev(*lv.live, kKB) * kKB);
  // bands of eight B tiles, a band's A tiles one after the other, a contiguous
  // eighth to each XCD
  const int item = xcd_item(blockIdx.x, ta * tb * slices);
  if (item < 0) return;
  const int zi = item / (ta * tb), it = item % (ta * tb);
  const int band = it / (kBand * ta), in = it % (kBand * ta), bw = min(kBand, tb - band * kBand);
  const int a0 = in / bw * SH::BA, b0 = (band * kBand + in % bw) * SH::BB;
  const int klo = zi * kchunk, nst = max(0, (min(K, klo + kchunk) - klo + kKB - 1) / kKB);

  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, r = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6), wa = w % SH::WA, wb = w / SH::WA;
  typename OA::template Tile<SH::BA, SH::T> la;
  typename OB::template Tile<SH::BB, SH::T> lb;
  typename OA::template Frag<SH::BA> fa;
  typename OB::template Frag<SH::BB> fb;
  la.init(oa, a0, tid);
  lb.init(ob, b0, tid);
  fa.init(wa * 16 * FA, g, r);
  fb.init(wb * 16 * FB, g, r);
  v4f acc[FA][FB];
  zero_acc(acc);
  constexpr int kCopies = decltype(la)::kCopies + decltype(lb)::kCopies;
  const uint32_t dst = __builtin_amdgcn_readfirstlane(
      lds_addr_of(reinterpret_cast<const float*>(lds)) + 1024u * w);
  auto issue = [&](int st) {
    const uint32_t d = dst + (st % S) * SH::kStage;
    la.issue(klo + st * kKB, d);
    lb.issue(klo + st * kKB, d + SH::BA * 128);
  };
#pragma unroll
  for (int st = 0; st < S - 1; ++st)
    if (st < nst) issue(st);
  for (int st = 0; st < nst; ++st) {
    // this stage has landed and the one before it has been read, everywhere
    if (st + S - 2 < nst) wait_vmcnt_lgkm0<(S - 2) * kCopies>();
    else wait_vmcnt_lgkm0<0>();
    barrier_nofence();
    if (st + S - 1 < nst) issue(st + S - 1);
    const char* A = lds + (st % S) * SH::kStage;
    const char* B = A + SH::BA * 128;
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      bf16x8 a[FA], b[FB];
#pragma unroll
      for (int f = 0; f < FB; ++f) b[f] = fb.read(B, kk, f);
#pragma unroll
      for (int f = 0; f < FA; ++f) a[f] = fa.read(A, kk, f);
#pragma unroll
      for (int i = 0; i < FA; ++i)
#pragma unroll
        for (int j = 0; j < FB; ++j) acc[i][j] = mfma_bf16_16x16x32(a[i], b[j], acc[i][j]);
    }
  }
  ep.template operator()<SH>(lds, zi, a0 + wa * 16 * FA, b0 + wb * 16 * FB, w, g, r, acc);
}

template <class SH, class OA, class OB, class EP>
void product(const char* name, OA oa, OB ob, EP ep, Live lv, int ma, int mb, int K, int kchunk,
             hipStream_t s) {
  const int ta = cdiv(ma, SH::BA), tb = cdiv(mb, SH::BB), slices = cdiv(K, kchunk);
  CAVS_LAUNCH(name, (k_vocab_bf<SH, OA, OB, EP>), dim3(xcd_grid(ta * tb * slices)), dim3(SH::T), 0, s,
              oa, ob, ep, lv, ta, tb, K, kchunk, slices);
}

// Words are the tile's A rows: lane (g, r) holds words 16 f + 4 g .. + 3 of its
// row r of each group of 16.
template <bool LOSS, bool TEACH>
struct BfVocab {
  VocabEp e;
  template <class SH>
  __device__ void operator()(char* lds, int, int a, int b, int w, int g, int r,
                             const v4f (&acc)[SH::FA][SH::FB]) const {
    constexpr int NC = 16 * SH::FA, NV = NC / 4;
    static_assert(SH::T / 64 * kSlabFloats<NC> * 4 <= SH::kBytes, "slabs fit the stages' LDS");
    static_assert(LOSS || NC % 64 == 0, "whole lanes of column sums");
    const int a0 = e.col0 + a;
    auto col = [](int i, int gg) { return 16 * (i >> 2) + 4 * gg + (i & 3); };
    float bias[NV], db[NC / 64] = {};
    vocab_bias(e, a0, g, col, bias);
    if (!LOSS || TEACH) __syncthreads();   // the slabs take the stages' place
    float* slab = reinterpret_cast<float*>(lds) + w * kSlabFloats<NC>;
    const int live = *e.live;
#pragma unroll
    for (int f = 0; f < SH::FB; ++f) {
      float z[NV];
#pragma unroll
      for (int i = 0; i < NV; ++i) z[i] = acc[i >> 2][f][i & 3] + bias[i];
      vocab_rows16<LOSS, TEACH, u16, NC>(e, z, col, b + 16 * f, 1, a0, a0 / NC, live, slab, db);
    }
    if (!LOSS) {
#pragma unroll
      for (int k = 0; k < NC / 64; ++k)
        e.dbp[(size_t)(b / (16 * SH::FB)) * e.ldz + a + (threadIdx.x & 63) + 64 * k] = db[k];
    }
  }
};

// rows of the output are the B rows, its columns the A rows
struct BfOut {
  VocabOut o;
  template <class SH>
  __device__ void operator()(char*, int z, int a, int b, int, int g, int r,
                             const v4f (&acc)[SH::FA][SH::FB]) const {
    const float w = o.scale ? *o.scale : 1.f;
#pragma unroll
    for (int j = 0; j < SH::FB; ++j)
#pragma unroll
      for (int i = 0; i < SH::FA; ++i)
        vocab_store4(o, w, z, b + 16 * j + r, a + 16 * i + 4 * g,
                     make_float4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]));
  }
};

using Big = Shape<2, 4, 8, 4, 2>;    // 256 x 256, eight wavefronts, 128 KB

template <bool LOSS>
void logits(const char* name, const VocabNet& v, int col0, int cols, hipStream_t s) {
  const ColsOp w{(const u16*)v.Ws + col0, v.ldw, v.Cq - col0};
  const RowsOp h{(const u16*)v.hp, v.H, v.rows, v.H};
  const VocabEp e = vocab_ep(v, col0);
  const Live lv{v.live, 1};
  if (v.K > 0) product<Big>(name, w, h, BfVocab<LOSS, true>{e}, lv, cols, v.rows, v.H, v.H, s);
  else product<Big>(name, w, h, BfVocab<LOSS, false>{e}, lv, cols, v.rows, v.H, v.H, s);
}

}  // namespace

void vocab_bf_loss(const VocabNet& v, hipStream_t s) {
  logits<true>("k_vocab_bf<loss>", v, 0, v.C, s);
}

void vocab_bf_dz(const VocabNet& v, int col0, int cols, hipStream_t s) {
  logits<false>("k_vocab_bf<dz>", v, col0, cols, s);
}

void vocab_bf_dh(const VocabNet& v, int col0, int cols, hipStream_t s) {
  const int K = cdiv(std::min(cols, v.C - col0), kKB) * kKB, kchunk = cdiv(K / kKB, v.Sh) * kKB;
  const VocabOut o{v.hpart, v.H, (size_t)v.rows * v.H, v.rows, v.H, 0, col0 > 0, nullptr};
  product<Big>("k_vocab_bf<dh>", RowsOp{(const u16*)v.Ws + col0, v.ldw, v.H, v.Cq - col0},
               RowsOp{(const u16*)v.dZ, v.P, v.rows, v.P}, BfOut{o}, Live{v.live, 1}, v.H, v.rows, K,
               kchunk, s);
}

void vocab_bf_dw(const VocabNet& v, int col0, int cols, const VocabOut& o, hipStream_t s) {
  const int kchunk = cdiv(v.rows / kKB, v.Sw) * kKB;
  product<Big>("k_vocab_bf<dw>", ColsOp{(const u16*)v.dZ, v.P, v.P},
               ColsOp{(const u16*)v.hp, v.H, v.H}, BfOut{o}, Live{v.live, 2}, cols, v.H, v.rows,
               kchunk, s);
}

}  // namespace cavs
