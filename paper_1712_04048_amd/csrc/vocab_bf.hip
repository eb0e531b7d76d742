// bf16 products of the vocabulary head: operands in bf16 in memory, copied
// straight to LDS (global_load_lds_dwordx4), fp32 accumulation on
// v_mfma_f32_16x16x32_bf16.
#include <algorithm>
#include <type_traits>

#include "lds_ring.h"
#include "vocab.h"
#include "xcd_map.h"

namespace cavs {
namespace {

constexpr int kKB = 64;   // parts of a contraction are multiples of this,
constexpr int kCK = 32;   // in chunks of this depth: one matrix instruction's

// An operand's tile of ROWS rows, kCK deep, in LDS, and how it gets there.  A
// workgroup's copy instruction moves 16 bytes per thread, thread t of T to byte
// 16 t, so the swizzles permute what a thread reads, not where it writes.
//
// Contiguous in the contraction: LDS rows of 64 bytes, their four 16-byte quads
// at quad ^ (row >> 2 & 3); eight lanes that read one quad of eight rows then
// cover the banks once.  The last quads may lie past the operand's end (kmax):
// they read its last ones instead, which meet zeros of the other operand.
struct RowsOp {
  const u16* p;
  long long ld;
  int rows, kmax;
  static constexpr int kReads = 1;   // LDS reads of a fragment
  static __device__ constexpr int quad(int row, int q) { return q ^ ((row >> 2) & 3); }
  template <int ROWS, int T>
  struct Tile {
    static constexpr int kCopies = ROWS * 64 / (16 * T);
    static_assert(kCopies * 16 * T == ROWS * 64, "whole copies");
    const u16* base[kCopies];
    int k, kmax;
    __device__ void init(const RowsOp& o, int r0, int tid) {
      kmax = o.kmax - 8;
#pragma unroll
      for (int i = 0; i < kCopies; ++i)
        base[i] = o.p + (size_t)min(r0 + ((i * T + tid) >> 2), o.rows - 1) * o.ld;
      k = 8 * quad(tid >> 2, tid & 3);   // T is a multiple of 64: the same for every i
    }
    __device__ void issue(int k0, uint32_t lds) const {
      const int kk = min(k0 + k, kmax);
#pragma unroll
      for (int i = 0; i < kCopies; ++i)
        copy16_to_lds(reinterpret_cast<const float*>(base[i] + kk), lds + 16 * T * i);
    }
  };
  // rows w0 + 16 f + r, k = 8 g ..
  template <int ROWS>
  struct Frag {
    uint32_t at;
    __device__ void init(int w0, int g, int r) { at = (w0 + r) * 64 + 16 * quad(r, g); }
    __device__ bf16x8 read(const char* lds, int f) const {
      return *reinterpret_cast<const bf16x8*>(lds + at + f * 1024);
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
  static constexpr int kReads = 2;
  static __device__ constexpr int swizzle(int k) { return (k & 3) | ((k >> 3) & 1) << 2; }
  template <int ROWS, int T>
  struct Tile {
    static_assert(ROWS >= 128, "eight segments to permute");
    static constexpr int kCopies = ROWS * 64 / (16 * T);
    static_assert(kCopies * 16 * T == ROWS * 64, "whole copies");
    const u16* base[kCopies];
    long long ld;
    __device__ void init(const ColsOp& o, int c0, int tid) {
      ld = o.ld;
#pragma unroll
      for (int i = 0; i < kCopies; ++i) {
        const int at = i * T + tid, k = at / (ROWS / 8), q = at % (ROWS / 8);
        const int c = c0 + 16 * ((q >> 1) ^ swizzle(k)) + 8 * (q & 1);
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
    __device__ bf16x8 read(const char* lds, int f) const {
      typedef short s4 __attribute__((ext_vector_type(4)));
      typedef short s8 __attribute__((ext_vector_type(8)));
      typedef __attribute__((address_space(3))) s4 lds_s4;
      const char* a = lds + at + (((seg0 + f) ^ s) << 5);
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
  // uniform, which the compiler does not see past another product's copies
  __device__ int tiles(int of) const { return cdiv_dev(__builtin_amdgcn_readfirstlane(*live), of); }
};

// A workgroup of WA x WB wavefronts: A rows 16 FA WA, B rows 16 FB WB, each
// wavefront 16 FA x 16 FB.  A ring of four chunks in LDS: a chunk's copies go out
// four chunks ahead of its products, and its fragments are read from LDS while
// the chunk before it is multiplied (the two sets of fragments and the sums take
// the registers that two wavefronts a SIMD leave).  One barrier a chunk.
template <int WA_, int WB_, int FA_, int FB_>
struct Shape {
  static constexpr int WA = WA_, WB = WB_, FA = FA_, FB = FB_, S = 4;
  static constexpr int T = 64 * WA * WB, BA = 16 * FA * WA, BB = 16 * FB * WB;
  static constexpr int kStage = (BA + BB) * 64, kBytes = S * kStage;
  static constexpr int kWgs = 8 / (WA * WB);   // that share a CU, two wavefronts a SIMD
};

constexpr int kBand = 8;

// One product: A rows ta tiles, B rows tb tiles, the contraction in `slices`
// parts of kchunk.
template <class SH, class OA, class OB, class EP>
struct Product {
  using Own = typename EP::template Own<SH>;
  OA oa;
  OB ob;
  EP ep;
  Live lv;
  int ta, tb, K, kchunk, slices;

  Product(OA a, OB b, EP e, Live l, int ma, int mb, int K_, int kchunk_)
      : oa(a), ob(b), ep(e), lv(l), ta(cdiv(ma, SH::BA)), tb(cdiv(mb, SH::BB)), K(K_), kchunk(kchunk_),
        slices(cdiv(K_, kchunk_)) {}
  int grid() const { return xcd_grid(ta * tb * slices); }

  // Workgroup `at` of XCD x among this product's, or at less their number and
  // false.  A contiguous eighth of the items to each XCD, in bands of eight B
  // tiles, a band's A tiles one after the other.
  __device__ __forceinline__ bool take(int x, int& at, char* lds) const {
    at = __builtin_amdgcn_readfirstlane(at);   // uniform, as in Live
    const int tb_ = lv.what == 1 ? lv.tiles(SH::BB) : tb;
    const int items = ta * tb_ * slices, per = (items + 7) / 8, item = x * per + at;
    if (at >= per) {
      at -= per;
      return false;
    }
    if (item < items) {
      const int zi = item / (ta * tb_), it = item % (ta * tb_);
      const int band = it / (kBand * ta), in = it % (kBand * ta), bw = min(kBand, tb_ - band * kBand);
      run(lds, zi, in / bw * SH::BA, (band * kBand + in % bw) * SH::BB);
    }
    return true;
  }

  __device__ __forceinline__ void run(char* lds, int zi, int a0, int b0) const {
    constexpr int FA = SH::FA, FB = SH::FB, S = SH::S;
    const int end = lv.what == 2 ? min(K, lv.tiles(kKB) * kKB) : K;
    const int klo = __builtin_amdgcn_readfirstlane(zi * kchunk);
    // an even number of chunks
    const int nc = __builtin_amdgcn_readfirstlane(max(0, (min(end, klo + kchunk) - klo + kKB - 1) / kKB) * 2);
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
    auto issue = [&](int c) {
      const uint32_t d = __builtin_amdgcn_readfirstlane(dst + (c % S) * SH::kStage);
      la.issue(klo + c * kCK, d);
      lb.issue(klo + c * kCK, d + SH::BA * 64);
    };
    struct Set {
      bf16x8 a[FA], b[FB];
    } set[2];
    auto read = [&](Set& x, int c) {
      const char* A = lds + (c % S) * SH::kStage;
#pragma unroll
      for (int f = 0; f < FB; ++f) x.b[f] = fb.read(A + SH::BA * 64, f);
#pragma unroll
      for (int f = 0; f < FA; ++f) x.a[f] = fa.read(A, f);
    };
#pragma unroll
    for (int c = 0; c < S; ++c)
      if (c < nc) issue(c);
    ep.template prepare<SH>(lds + SH::kBytes, a0, b0);   // before the first barrier
    if (nc > 0) {
      if (nc >= S) wait_vmcnt_lgkm0<(S - 1) * kCopies>();
      else wait_vmcnt_lgkm0<0>();
      barrier_nofence();
      read(set[0], 0);
    }
    for (int c0 = 0; c0 < nc; c0 += 2) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int c = c0 + h;
        // the next chunk has landed, and this one's fragments have been read,
        // everywhere: its place is free
        if (c + S - 1 < nc) wait_vmcnt_lgkm0<(S - 2) * kCopies>();
        else wait_vmcnt_lgkm0<0>();
        barrier_nofence();
        if (c + S < nc) issue(c + S);
        read(set[1 - h], c + 1);   // past the last chunk: a stale one, not used
        const Set& x = set[h];
#pragma unroll
        for (int i = 0; i < FA; ++i)
#pragma unroll
          for (int j = 0; j < FB; ++j) acc[i][j] = mfma_bf16_16x16x32(x.a[i], x.b[j], acc[i][j]);
        constexpr int kReads = OA::kReads * FA + OB::kReads * FB, kPer = FA * FB / kReads > 0 ? FA * FB / kReads : 1;
#pragma unroll
        for (int i = 0; i < kReads; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);      // an LDS read
          __builtin_amdgcn_sched_group_barrier(0x008, kPer, 0);   // products
        }
        __builtin_amdgcn_sched_group_barrier(0x008, FA * FB, 0);
      }
    }
    ep.template operator()<SH>(lds + SH::kBytes, zi, a0, b0, wa, wb, g, r, acc);
  }
};

// One or more independent products, the workgroups of the first ones first.
template <class SH, class... P>
__global__ void __launch_bounds__(SH::T, 2) k_vocab_bf(P... p) {
  // an empty struct has a size of 1, and a workgroup of 80 KB + 1 a CU to itself
  // (dL/dh of 64 rows, 32 000 words, H = 2048: 42 us, two a CU 38)
  constexpr size_t kOwn = std::max({std::is_empty_v<typename P::Own> ? 0 : sizeof(typename P::Own)...});
  static_assert(SH::kBytes + kOwn <= 160 * 1024 / SH::kWgs, "workgroups that share a CU");
  __shared__ __attribute__((aligned(16))) char lds[SH::kBytes + kOwn];
  const int x = blockIdx.x & 7;
  int at = blockIdx.x >> 3;
  (void)(p.take(x, at, lds) || ...);
}

template <class SH, class... P>
void launch(const char* name, hipStream_t s, P... p) {
  CAVS_LAUNCH(name, (k_vocab_bf<SH, P...>), dim3((p.grid() + ...)), dim3(SH::T), 0, s, p...);
}

// Words are the tile's A rows: lane (g, r) holds words 16 f + 4 g .. + 3 of its
// row r of each group of 16.  dz with a teacher needs 14 registers more than there
// are beside the sums: they go through scratch in the epilogue, 14 stores and 43
// loads of a lane each tile; the products spill nothing, nor do the other epilogues.
template <bool LOSS, bool TEACH>
struct BfVocab {
  VocabEp e;
  // The tile's words' biases and rows' constants, in LDS beside the stages: asked
  // for with the first stage's copies, they have come long before the epilogue,
  // which one workgroup a CU leaves nothing else to run in.
  template <class SH>
  struct Own {
    float bias[SH::BA];
    float4 c[LOSS ? 1 : SH::BB];
    int label[SH::BB];
    uint32_t range[TEACH ? SH::WA : 1][SH::BB];
  };
  template <class SH>
  __device__ void prepare(char* own, int a, int b) const {
    Own<SH>& o = *reinterpret_cast<Own<SH>*>(own);
    constexpr int NC = 16 * SH::FA;
    const int live = *e.live;
    for (int i = threadIdx.x; i < SH::BA; i += SH::T) {
      const int c = e.col0 + a + i;
      o.bias[i] = c < e.C ? (e.bs ? e.bs[c] : 0.f) : -INFINITY;
    }
    for (int i = threadIdx.x; i < SH::BB; i += SH::T) {
      const VocabRow v = vocab_row<LOSS, false>(e, b + i, 0, live);
      if (!LOSS) o.c[i] = v.c;
      o.label[i] = v.label;
      if (TEACH)
        for (int k = 0; k < SH::WA; ++k)
          o.range[k][i] = b + i < live ? e.trange[(size_t)((e.col0 + a) / NC + k) * e.rows + b + i] : 0u;
    }
  }
  template <class SH>
  __device__ void operator()(const char* own, int, int ta, int tb, int wa, int wb, int g, int r,
                             const v4f (&acc)[SH::FA][SH::FB]) const {
    const Own<SH>& o = *reinterpret_cast<const Own<SH>*>(own);
    constexpr int NC = 16 * SH::FA, NV = NC / 4;
    const int a = ta + wa * NC, b = tb + wb * 16 * SH::FB, a0 = e.col0 + a;
    auto col = [](int i, int gg) { return 16 * (i >> 2) + 4 * gg + (i & 3); };
    float db[NV] = {};
#pragma unroll
    for (int f = 0; f < SH::FB; ++f) {
      float z[NV];
#pragma unroll
      for (int i = 0; i < NV; i += 4) {
        const float4 x = *reinterpret_cast<const float4*>(o.bias + wa * NC + col(i, g));
        z[i] = acc[i >> 2][f][0] + x.x;
        z[i + 1] = acc[i >> 2][f][1] + x.y;
        z[i + 2] = acc[i >> 2][f][2] + x.z;
        z[i + 3] = acc[i >> 2][f][3] + x.w;
      }
      const int at = wb * 16 * SH::FB + 16 * f + r, row = tb + at;
      const VocabRow v{LOSS ? f4zero() : o.c[LOSS ? 0 : at], o.label[at], TEACH ? o.range[TEACH ? wa : 0][at] : 0u};
      vocab_rows16<LOSS, TEACH, u16, NC>(e, z, col, row, v, a0, (size_t)(a0 / NC) * e.rows + row, db);
    }
    if (!LOSS) vocab_db<NC>(e, db, col, a0, b / (16 * SH::FB));
  }
};

// rows of the output are the B rows, its columns the A rows
struct BfOut {
  VocabOut o;
  template <class SH>
  struct Own {};
  template <class SH>
  __device__ void prepare(char*, int, int) const {}
  template <class SH>
  __device__ void operator()(const char*, int z, int ta, int tb, int wa, int wb, int g, int r,
                             const v4f (&acc)[SH::FA][SH::FB]) const {
    const int a = ta + wa * 16 * SH::FA, b = tb + wb * 16 * SH::FB;
    const float w = o.scale ? *o.scale : 1.f;
#pragma unroll
    for (int j = 0; j < SH::FB; ++j)
#pragma unroll
      for (int i = 0; i < SH::FA; ++i)
        vocab_store4(o, w, z, b + 16 * j + r, a + 16 * i + 4 * g,
                     make_float4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]));
  }
};

// The loss of few rows or words: 128 words x 64 rows to a workgroup (four
// wavefronts of 32 x 64), two stages of W_s's columns in flight in registers; of
// few rows it is bound by reading them (4 x 50 000 x 1024: 24 us, 4.3 TB/s; 4 x 128
// 000 x 2048: 97 us, 5.4 TB/s).  They
// come from W_s as it is, whatever C is: a 16-byte load needs no more than the
// alignment of its elements, where the copies to LDS want four bytes (padding
// 50 001 columns took 53 of 140 us).
// FB: groups of 16 rows.  Of at most 16 rows one alone: the products and reads of
// h of the other three took 27 us instead of 24 of 4 x 50 000 x 1024, 111 instead of
// 97 of the larger.
constexpr int kFewRows = kVocabFew, kFewWords = 128;
template <bool TEACH, int FB>
__global__ void __launch_bounds__(256, 2) k_vocab_few(VocabEp e, const u16* __restrict__ W,
                                                      const u16* __restrict__ hp, int H) {
  constexpr int FA = 2, kA = kFewWords * 128, kB = 16 * FB * 128;
  __shared__ __attribute__((aligned(16))) char lds[2][kA + kB];
  __shared__ float stats[3][4][kFewRows];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, g = lane >> 4, r = lane & 15;
  const int a0 = blockIdx.x * kFewWords, row0 = blockIdx.y * kVocabFew, C = e.C;
  if (row0 >= *e.live) return;
  const size_t end = (size_t)H * C;   // at least 64 values
  // a stage is two chunks, in LDS as ColsOp and RowsOp have them
  int ka[4], ca[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int at = (i & 1) * 256 + tid, q = at & 15, k = at >> 4;
    ka[i] = kCK * (i >> 1) + k;
    ca[i] = a0 + 16 * ((q >> 1) ^ ColsOp::swizzle(k)) + 8 * (q & 1);
  }
  const u16* hb = hp + (size_t)(row0 + (tid >> 2)) * H + 8 * RowsOp::quad(tid >> 2, tid & 3);
  struct Stage {
    uint4 a[4], b[2];
  } st[2];
  auto load = [&](Stage& x, int k0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x.a[i] = vocab_load8(W, (size_t)(k0 + ka[i]) * C + ca[i], end);
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (FB == 4 || tid < 64 * FB) x.b[i] = *reinterpret_cast<const uint4*>(hb + k0 + kCK * i);
  };
  ColsOp::Frag<kFewWords> fa;
  RowsOp::Frag<kFewRows> fb;
  fa.init(32 * w, g, r);
  fb.init(0, g, r);
  v4f acc[FA][FB];
  zero_acc(acc);
  load(st[0], 0);
  load(st[1], min(kKB, H - kKB));
  for (int k0 = 0; k0 < H; k0 += 2 * kKB) {
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      if (k0 + s * kKB >= H) break;
      char* L = lds[s];
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(L + 16 * (i * 256 + tid)) = st[s].a[i];
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (FB == 4 || tid < 64 * FB) *reinterpret_cast<uint4*>(L + kA + i * (kB / 2) + 16 * tid) = st[s].b[i];
      __syncthreads();   // the other buffer's readers are past this one's barrier
      load(st[s], min(k0 + (s + 2) * kKB, H - kKB));   // past the end: the last stage, unused
      __builtin_amdgcn_sched_barrier(0);   // the loads go out before these products
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        bf16x8 a[FA], b[FB];
#pragma unroll
        for (int f = 0; f < FA; ++f) a[f] = fa.read(L + kk * (kA / 2), f);
#pragma unroll
        for (int f = 0; f < FB; ++f) b[f] = fb.read(L + kA + kk * (kB / 2), f);
#pragma unroll
        for (int i = 0; i < FA; ++i)
#pragma unroll
          for (int j = 0; j < FB; ++j) acc[i][j] = mfma_bf16_16x16x32(a[i], b[j], acc[i][j]);
      }
    }
  }
  vocab_few_end<TEACH, kFewWords, FB>(e, stats, a0, row0, [&](int i, int f) { return acc[i >> 2][f][i & 3]; });
}

using Big = Shape<2, 4, 8, 4>;    // 256 x 256, eight wavefronts, 128 KB
using Few = Shape<4, 1, 4, 4>;    // 256 x 64, four wavefronts, 80 KB: two share a CU

template <bool LOSS, bool TEACH>
using Logits = Product<Big, ColsOp, RowsOp, BfVocab<LOSS, TEACH>>;
template <bool LOSS, bool TEACH>
Logits<LOSS, TEACH> logits(const VocabNet& v, int col0, int cols) {
  return {ColsOp{(const u16*)v.Ws + col0, v.ldw, v.Cq - col0}, RowsOp{(const u16*)v.hp, v.H, v.rows, v.H},
          BfVocab<LOSS, TEACH>{vocab_ep(v, col0)}, Live{v.live, 1}, cols, v.rows, v.H, v.H};
}

template <class SH>
Product<SH, RowsOp, RowsOp, BfOut> dh(const VocabNet& v, int col0, int cols) {
  const int K = cdiv(cols, kKB) * kKB, kchunk = cdiv(K / kKB, v.Sh) * kKB;
  const VocabOut o{v.hpart, v.H, (size_t)v.rows * v.H, v.rows, v.H, 0, col0 > 0, nullptr};
  return {RowsOp{(const u16*)v.Ws + col0, v.ldw, v.H, v.Cq - col0},
          RowsOp{(const u16*)vocab_dz_at(v, col0), v.P, v.rows, v.P}, BfOut{o}, Live{v.live, 1}, v.H, v.rows, K, kchunk};
}

Product<Big, ColsOp, ColsOp, BfOut> dw(const VocabNet& v, int col0, int cols, const VocabOut& o) {
  return {ColsOp{(const u16*)vocab_dz_at(v, col0), v.P, v.P}, ColsOp{(const u16*)v.hp, v.H, v.H}, BfOut{o},
          Live{v.live, 2}, cols, v.H, cdiv(v.n, kKB) * kKB, cdiv(cdiv(v.n, kKB), v.Sw) * kKB};
}

}  // namespace

void vocab_bf_loss(const VocabNet& v, const void* W, hipStream_t s) {
  if (v.small) {
    const dim3 grid(cdiv(v.C, kFewWords), cdiv(v.n, kVocabFew));
    const VocabEp e = vocab_ep(v, 0);
    auto go = [&](auto* kernel) {
      CAVS_LAUNCH("k_vocab_few", kernel, grid, dim3(256), 0, s, e, (const u16*)W, (const u16*)v.hp, v.H);
    };
    if (v.n <= 16) v.K > 0 ? go(k_vocab_few<true, 1>) : go(k_vocab_few<false, 1>);
    else v.K > 0 ? go(k_vocab_few<true, 4>) : go(k_vocab_few<false, 4>);
    return;
  }
  vocab_launches(v, [&](int col0, int cols) {
    if (v.K > 0) launch<Big>("k_vocab_bf<loss>", s, logits<true, true>(v, col0, cols));
    else launch<Big>("k_vocab_bf<loss>", s, logits<true, false>(v, col0, cols));
  });
}

void vocab_bf_dz(const VocabNet& v, int col0, int cols, hipStream_t s) {
  if (v.K > 0) launch<Big>("k_vocab_bf<dz>", s, logits<false, true>(v, col0, cols));
  else launch<Big>("k_vocab_bf<dz>", s, logits<false, false>(v, col0, cols));
}

// next > 0: the columns of the next piece, whose dz is formed beside this one's
// products (it fills the CUs that they leave: 196 tiles of dW_s and 112 of dL/dh
// take turns on 256 CUs badly by themselves).
void vocab_bf_grads(const VocabNet& v, int col0, int cols, int next, const VocabOut& o, hipStream_t s) {
  const auto w = dw(v, col0, cols, o);
  if (v.few) {
    launch<Big>("k_vocab_bf<dw>", s, w);
    launch<Few>("k_vocab_bf<dh, few>", s, dh<Few>(v, col0, cols));
  } else {
    // the longer items first, the next piece's short ones last
    const auto h = dh<Big>(v, col0, cols);
    auto with = [&](auto first, auto second) {
      if (next == 0) launch<Big>("k_vocab_bf<dw, dh>", s, first, second);
      else if (v.K > 0)
        launch<Big>("k_vocab_bf<dw, dh, dz>", s, first, second, logits<false, true>(v, col0 + cols, next));
      else launch<Big>("k_vocab_bf<dw, dh, dz>", s, first, second, logits<false, false>(v, col0 + cols, next));
    };
    if (w.kchunk >= h.kchunk) with(w, h);
    else with(h, w);
  }
}

}  // namespace cavs
