// The vocabulary head: the live rows, the teacher's distributions, the
// softmax statistics joined over the vocabulary, the loss, and the order of the
// products (vocab_x3.hip, vocab_bf.hip).
//
//   loss       z = h W_s + b_s tile by tile; a tile leaves each row's largest z
//              and sum of exponentials over its words, not z itself
//   gradient   for each piece of P words: z again, dz from the joined
//              statistics into dZ [rows, P], then dW_s of the piece = h^T dZ and
//              dL/dh += dZ W_s^T
// The second pass over z costs two of eight units of work; what it saves is
// rows x C values of memory (the head inside cavs_forward keeps them).  Where one
// piece is the whole vocabulary, z is kept in it instead if that is faster.
#include <math.h>

#include <algorithm>

#include "vocab.h"

namespace cavs {
namespace {

constexpr size_t kPieceBytes = (size_t)256 << 20;   // of dZ
constexpr size_t kKeepBytes = (size_t)96 << 20;     // of z in bf16, see vocab_net
// Sizes whose tiles and offsets the kernels count in 32 bits.
constexpr int kVocabMaxRows = 1 << 20, kVocabMaxWords = 1 << 20, kVocabMaxH = 1 << 15;
static_assert(kPieceBytes / (kVocabFew * 4) >= kVocabMaxWords,
              "few rows are one piece, whose z is kept: their buffers end before a tile of 256 rows");

// The live rows: their list and numbering, their labels, their rows of h in the
// products' type (zeros behind the last), and unit / their number.
// A workgroup takes R of the caller's rows and counts the labels before them
// itself, so that nothing waits for a list: R is at least 16 and at least n /
// 512, which bounds what all of them read to 512 n labels.
template <class IN, class OUT>
__global__ void __launch_bounds__(256) k_vocab_rows(VocabNet v, int R, const int* __restrict__ label,
                                                    float* row_loss, int* err) {
  __shared__ int wsum[4], src_of[64], found;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, n = v.n, C = v.C, H = v.H;
  const int lo = blockIdx.x * R, hi = min(lo + R, n);
  int before = 0;
  if (label) {   // lo is a multiple of 4
#pragma unroll 4
    for (int i = 4 * tid; i < lo; i += 1024) {
      int y[4];
      __builtin_memcpy(y, label + i, 16);
#pragma unroll
      for (int k = 0; k < 4; ++k) before += (unsigned)y[k] < (unsigned)C;
    }
  } else if (tid == 0) {
    before = lo;
  }
  before = wave_sum_int(before);
  if (lane == 0) wsum[w] = before;
  __syncthreads();
  before = wsum[0] + wsum[1] + wsum[2] + wsum[3];
  bool bad = false;
  // 64 rows at a time: the first wavefront numbers them, then all copy
  for (int i0 = lo; i0 < hi; i0 += 64) {
    if (w == 0) {
      const int i = i0 + lane;
      const int y = i < hi ? (label ? label[i] : 0) : -1;
      const bool on = y >= 0 && y < C;
      bad |= y < -1 || y >= C;
      const unsigned long long m = __ballot(on);
      const int k = __popcll(m & ((1ull << lane) - 1)), at = before + k;
      if (i < hi) v.place[i] = on ? at : -1;
      if (on) {
        src_of[k] = i;
        v.rows_list[at] = i;
        v.label[at] = label ? y : -1;
      } else if (i < hi && row_loss) {
        row_loss[i] = 0.f;
      }
      if (lane == 0) found = __popcll(m);
    }
    __syncthreads();
    const int nf = found;
    constexpr int VEC = 8;
    const int q = H / VEC, items = nf * q;   // H is a multiple of 64
#pragma unroll 4
    for (int x = tid; x < items; x += 256) {
      const int k = (unsigned)x / (unsigned)q, c = (x - k * q) * VEC;
      float val[VEC];
      load_row<VEC>((const IN*)v.h + (size_t)src_of[k] * H + c, val);
      store_row<VEC>((OUT*)v.hp + (size_t)(before + k) * H + c, val);
    }
    before += nf;
    __syncthreads();
  }
  if (bad) err[1] = 1;
  if (hi < n) return;
  if (tid < 64) v.zrow[tid] = 0.f;
  if (tid == 0) {
    *v.live = before;
    *v.scal = v.unit / (float)max(before, 1);
  }
  // Zeros as far as they can meet a live row's: to the end of a chunk of dW_s's
  // contraction, and in fp32 of a tile (a NaN in it would have it formed again).
  // H is a multiple of 64: whole 16 bytes.
  const size_t from = (size_t)before * H * sizeof(OUT);
  const int tile = v.bf || v.few ? kVocabFew : 2 * kVocabFew;
  const size_t to = (size_t)cdiv_dev(before, tile) * tile * H * sizeof(OUT);
  for (size_t o = from + 16 * tid; o < to; o += 256 * 16) st4((float*)((char*)v.hp + o), f4zero());
}

// bf16 W_s with its rows padded to whole 16 bytes (zeros), for a C that is not:
// 16 bytes a thread, read at the alignment of an element.
__global__ void __launch_bounds__(256) k_vocab_pad(int H, int C, int Cq, const u16* __restrict__ W, u16* out) {
  const int c = (blockIdx.x * 256 + threadIdx.x) * 8;
  if (c >= C) return;
  const size_t row = blockIdx.y;
  *reinterpret_cast<uint4*>(out + row * Cq + c) = vocab_row8(W, row * C + c, (size_t)H * C, C - c);
}

// The teacher's distribution over its words of a live row, q = softmax(t / T)
// over the words that are there and have a logit above -inf, the words in
// ascending order and their ranges in the products' slots of words.  A word that
// is listed twice counts as the sum of its entries, at its first place; the
// loss's sum of q ln q is over the entries.  A wavefront per row; an entry's
// place is the number of smaller ones (K at most kVocabMaxK).
__global__ void __launch_bounds__(256) k_vocab_teacher(VocabNet v, const int* __restrict__ top_word,
                                                       const float* __restrict__ top_logit, int* err) {
  constexpr int PER = kVocabMaxK / 64, kNone = 0x7fffffff;
  __shared__ __attribute__((aligned(16))) int words[4][kVocabMaxK], sorted[4][kVocabMaxK];
  __shared__ __attribute__((aligned(16))) float qs[4][kVocabMaxK];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, row = blockIdx.x * 4 + w, K = v.K;
  if (row >= *v.live) return;
  const size_t src = (size_t)v.rows_list[row] * K, dst = (size_t)row * K;
  const float invT = 1.f / v.temp;
  int id[PER];
  float t[PER], m = -INFINITY;
  bool bad = false, nan = false;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    const int j = lane + 64 * k;
    const int x = j < K ? top_word[src + j] : -1;
    bad |= x < -1 || x >= v.C;
    id[k] = x >= 0 && x < v.C ? x : kNone;
    t[k] = id[k] != kNone ? top_logit[src + j] * invT : -INFINITY;
    nan |= t[k] != t[k];
    m = fmaxf(m, t[k]);
  }
  if (bad) err[1] = 1;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, kWave));
  const bool some = m > -INFINITY || __any(nan);   // a NaN is not nothing
  float sum = 0.f, q[PER], s = 0.f;
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    q[k] = t[k] == -INFINITY ? 0.f : expf(t[k] - m);
    sum += q[k];
  }
  sum = wave_sum(sum);
  const float ls = logf(sum);
#pragma unroll
  for (int k = 0; k < PER; ++k) {
    q[k] = some ? q[k] / sum : 0.f;
    if (some && !(q[k] == 0.f)) s += q[k] * (t[k] - m - ls);
    words[w][lane + 64 * k] = id[k];
    qs[w][lane + 64 * k] = q[k];
  }
  s = wave_sum(s);
  if (lane == 0) v.tsum[row] = make_float2(s, some ? 1.f : 0.f);
  wave_lds_fence();
  // four entries at a time against all of a lane's (one by one, an entry of theirs
  // after the other, 600 rows of 200 words took 70 us); entries past K are kNone
  auto rank = [&](auto reach) {
    constexpr int R = decltype(reach)::value;
    int place[R] = {};
    bool first[R];
    float total[R] = {};
#pragma unroll
    for (int k = 0; k < R; ++k) first[k] = true;
    for (int i0 = 0; i0 < K; i0 += 4) {
      const int4 x4 = *reinterpret_cast<const int4*>(words[w] + i0);
      const float4 q4 = *reinterpret_cast<const float4*>(qs[w] + i0);
      const int x[4] = {x4.x, x4.y, x4.z, x4.w};
      const float y[4] = {q4.x, q4.y, q4.z, q4.w};
#pragma unroll
      for (int k = 0; k < R; ++k)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const bool same = x[u] == id[k], before = same && i0 + u < lane + 64 * k;
          place[k] += x[u] < id[k] || before;
          first[k] = first[k] && !before;
          total[k] += same ? y[u] : 0.f;
        }
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
      if (lane + 64 * k >= K) continue;
      sorted[w][place[k]] = id[k];
      v.tword[dst + place[k]] = id[k];
      v.tq[dst + place[k]] = first[k] && id[k] != kNone ? total[k] : 0.f;
    }
  };
  if (K <= 64) rank(std::integral_constant<int, 1>{});
  else if (K <= 128) rank(std::integral_constant<int, 2>{});
  else rank(std::integral_constant<int, PER>{});
  wave_lds_fence();
  auto below = [&](long long word) {   // the row's words below this one
    int lo = 0, hi = K;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (sorted[w][mid] < word) lo = mid + 1;
      else hi = mid;
    }
    return lo;
  };
  // the last tile's slots past C as well; a slot ends where the next one begins
  const int slots = cdiv_dev(v.C, kVocabTile) * (kVocabTile / v.slot_words);
  for (int k0 = 0; k0 < slots; k0 += 63) {
    const int k = k0 + lane, from = below((long long)k * v.slot_words), to = __shfl_down(from, 1, kWave);
    if (lane < 63 && k < slots) v.trange[(size_t)k * v.rows + row] = from | (uint32_t)to << 16;
  }
}

// A live row's loss and what its dz is made from, from its joined statistics.
__device__ float vocab_row_end(const VocabNet& v, int row, float m, float s, float t, float dot,
                               float* row_loss) {
  float val = 0.f, has = 0.f;
  const float a = v.alpha;
  const int y = v.label[row];
  if (y >= 0 && a < 1.f) val = (1.f - a) * (logf(s) + (m - v.zlab[row]));
  if (v.K > 0) {
    const float2 q = v.tsum[row];
    has = q.y;
    if (has != 0.f && a > 0.f) val += a * v.temp * v.temp * (q.x + logf(t) + dot / v.temp);
  }
  v.val[row] = val;
  if (row_loss) row_loss[v.rows_list[row]] = val;
  // in units of v.unit
  const float lab = a < 1.f ? 1.f : 0.f, c1 = lab != 0.f ? 1.f / s : 0.f;
  const float cT = has != 0.f ? v.distw / t : 0.f;
  if (c1 == 0.f && cT == 0.f) m = INFINITY;   // no dz, as behind the last row
  v.rowc[row] = v.two ? make_float4(m, c1, cT, lab) : make_float4(m, c1 + cT, 0.f, lab);
  return val;
}

// A row's statistics joined over the slots, its loss, and what its dz is made
// from.  16 rows a workgroup, 64 lanes on every 64th slot (or teacher's word)
// of each, their sums added in their order.
//   CE = ln(sum exp(z - m)) + m - z_label
//   KD = T^2 (sum q ln q + ln(sum exp((z - m) / T)) + sum q (m - z) / T)
__global__ void __launch_bounds__(1024) k_vocab_join(VocabNet v, float* row_loss, float* loss) {
  __shared__ float sm[64][16], ss[64][16], st[64][16], sd[64][16];
  const int i = threadIdx.x & 15, k0 = threadIdx.x >> 4, row = blockIdx.x * 16 + i;
  const int nl = *v.live;
  const float4 none = make_float4(INFINITY, 0.f, 0.f, 0.f);   // exp(z - inf): no dz
  if ((int)blockIdx.x * 16 >= nl) {
    // the rest of the last tile of 256 rows
    if (k0 == 0 && (int)blockIdx.x * 16 < cdiv_dev(nl, kVocabTile) * kVocabTile) v.rowc[row] = none;
    if (loss && threadIdx.x == 0) *loss = 0.f;
    return;
  }
  // a thread's slots, eight at a time and all asked for before the first is used,
  // relative to the largest z so far
  constexpr int U = 8;
  float m = -INFINITY, s = 0.f, t = 0.f, dot = 0.f;
  auto at0 = [](float x) { return x == -INFINITY ? 0.f : x; };
  const float invT = 1.f / v.temp;
  for (int kk = k0; kk < v.slots; kk += 64 * U) {
    float pm[U], ps[U], pt[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const size_t at = (size_t)(kk + 64 * u) * v.rows + row;
      const bool there = kk + 64 * u < v.slots;
      pm[u] = there ? v.pm[at] : -INFINITY;
      ps[u] = there ? v.ps[at] : 0.f;
      pt[u] = there && v.two ? v.pt[at] : 0.f;
    }
    float mu = m;
#pragma unroll
    for (int u = 0; u < U; ++u) mu = fmaxf(mu, pm[u]);
    const float m0 = at0(mu), d0 = (m - m0) * kLog2e;
    s *= __builtin_amdgcn_exp2f(d0);
    t *= __builtin_amdgcn_exp2f(d0 * invT);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float d = (pm[u] - m0) * kLog2e;
      s += ps[u] * __builtin_amdgcn_exp2f(d);
      if (v.two) t += pt[u] * __builtin_amdgcn_exp2f(d * invT);
    }
    m = mu;
  }
  sm[k0][i] = m;
  __syncthreads();
  const float own = m;
#pragma unroll
  for (int k = 0; k < 64; ++k) m = fmaxf(m, sm[k][i]);
  const float d0 = (own - at0(m)) * kLog2e;
  s *= __builtin_amdgcn_exp2f(d0);
  t *= __builtin_amdgcn_exp2f(d0 * invT);
  if (row < nl)
    for (int j = k0; j < v.K; j += 64) {
      const size_t at = (size_t)row * v.K + j;
      const float q = v.tq[at];
      if (q != 0.f) dot += q * (m - v.ztop[at]);   // a word that is not there has none
    }
  ss[k0][i] = s;
  st[k0][i] = t;
  sd[k0][i] = dot;
  __syncthreads();
  if (k0 > 0) return;
  s = t = dot = 0.f;
#pragma unroll 16
  for (int k = 0; k < 64; ++k) {
    s += ss[k][i];
    t += st[k][i];
    dot += sd[k][i];
  }
  if (!v.two) t = s;
  float val = 0.f;
  if (row >= nl) v.rowc[row] = none;
  else val = vocab_row_end(v, row, m, s, t, dot, row_loss);
  if (!loss) return;
  // at most 16 rows, this the only workgroup: their mean, as vocab_mean adds it
  double sum = (double)val;
#pragma unroll
  for (int o = 8; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, kWave);
  if (i == 0) *loss = (float)(sum / (double)max(nl, 1));
}

// The mean of the live rows' losses, in 64 bits and a fixed order, by 256 threads.
__device__ void vocab_mean(const float* val, int nl, float* loss) {
  __shared__ double part[4];
  const int tid = threadIdx.x;
  double s = 0.0;
#pragma unroll 4
  for (int i = tid; i < nl; i += 256) s += (double)val[i];
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o, kWave);
  if ((tid & 63) == 0) part[tid >> 6] = s;
  __syncthreads();
  if (tid == 0) *loss = (float)((part[0] + part[1] + part[2] + part[3]) / (double)max(nl, 1));
}
__global__ void __launch_bounds__(256) k_vocab_mean(const float* __restrict__ val,
                                                    const int* __restrict__ live, float* loss) {
  vocab_mean(val, *live, loss);
}

// dz from the z that the loss kept (in place in fp32), as vocab_rows16 forms it,
// and its sums over 64 rows: 256 words x 64 rows a workgroup, a wavefront on
// whole rows of 1 KB.
// db: one group is all of db_s (else null, and the groups' sums go to dbp).
template <class OUT>
__global__ void __launch_bounds__(256) k_vocab_dz(VocabNet v, float* db_out) {
  __shared__ float4 sums[4][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nl = *v.live;
  const int c0 = blockIdx.x * 256, c = c0 + 4 * lane, r0 = blockIdx.y * 64;
  if (!db_out && r0 >= cdiv_dev(nl, kVocabTile) * kVocabTile) return;
  const float invT = 1.f / v.temp;
  // The teacher's words here of the wavefront's 16 rows: their ranges in one load, a
  // lane a word in another (one row after the other they are two dependent loads
  // each).  More than 64 are looked up row by row.
  int first = 0, there = 0, lo = 0, total = 0, tw = -1;
  float tq = 0.f;
  if (v.K > 0) {
    const int s0 = c0 / v.slot_words, s1 = s0 + 256 / v.slot_words - 1, row = r0 + 16 * w + (lane & 15);
    if (row < nl) {
      lo = v.trange[(size_t)s0 * v.rows + row] & 0xffffu;
      there = (int)(v.trange[(size_t)s1 * v.rows + row] >> 16) - lo;
    }
    int past = there;   // the sum up to a lane's row
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
      const int y = __shfl_up(past, o, 16);
      if ((lane & 15) >= o) past += y;
    }
    first = past - there;
    total = __builtin_amdgcn_readlane(past, 15);
    int k = 0;   // the row of word `lane` of them
#pragma unroll
    for (int i = 0; i < 15; ++i) k += __builtin_amdgcn_readlane(past, i) <= lane;
    const int j = __shfl(lo, k, kWave) + lane - __shfl(first, k, kWave);
    if (lane < total) {
      const size_t t = (size_t)(r0 + 16 * w + k) * v.K + j;
      tw = v.tword[t];
      tq = v.distw * v.tq[t];
    }
  }
  float4 db = f4zero();
#pragma unroll 4
  for (int rr = 0; rr < 16; ++rr) {
    const int row = __builtin_amdgcn_readfirstlane(r0 + 16 * w + rr);
    const size_t at = (size_t)row * v.P + c;
    float d[4] = {0.f, 0.f, 0.f, 0.f};
    if (row < nl) {
      const float4 z = ldg4(v.Z + at), k = v.rowc[row];
      const float x[4] = {z.x - k.x, z.y - k.x, z.z - k.x, z.w - k.x};
      const int lab = v.label[row];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        d[i] = k.y * __builtin_amdgcn_exp2f(x[i] * kLog2e);
        if (v.two) d[i] += k.z * __builtin_amdgcn_exp2f(x[i] * (invT * kLog2e));
        if (c + i == lab) d[i] -= k.w;
      }
      const int n = __builtin_amdgcn_readlane(there, rr), at0 = __builtin_amdgcn_readlane(first, rr);
      const size_t t0 = (size_t)row * v.K + __builtin_amdgcn_readlane(lo, rr);
      for (int j = 0; j < n; ++j) {
        int word;
        float q;
        if (total <= 64) {
          word = __builtin_amdgcn_readlane(tw, at0 + j);
          q = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(tq), at0 + j));
        } else {
          word = v.tword[t0 + j];
          q = v.distw * v.tq[t0 + j];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] -= c + i == word ? q : 0.f;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)   // no weights: no dz, whatever z is (vocab_rows16)
        d[i] = c + i < v.C && (k.y != 0.f || k.z != 0.f) ? d[i] : 0.f;
    }
    const float4 o = make_float4(d[0], d[1], d[2], d[3]);
    if constexpr (sizeof(OUT) == 2) st_bf4((u16*)v.dZ + at, o);
    else st4((float*)v.dZ + at, o);
    db = add4(db, o);
  }
  sums[w][lane] = db;
  __syncthreads();
  if (w > 0) return;
  db = add4(add4(sums[0][lane], sums[1][lane]), add4(sums[2][lane], sums[3][lane]));
  if (!db_out) {
    st4(v.dbp + (size_t)blockIdx.y * v.P + c, db);
    return;
  }
  const float x[4] = {db.x, db.y, db.z, db.w}, scale = *v.scal;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (c + i < v.C) db_out[c + i] = x[i] * scale;
}

// db_s of a piece: 64 columns a workgroup, its wavefronts every sixteenth group,
// their sums in order.
__global__ void __launch_bounds__(1024) k_vocab_db(int cols, int P, int group,
                                                   const int* __restrict__ live,
                                                   const float* __restrict__ dbp,
                                                   const float* __restrict__ scal, float* db) {
  __shared__ float sums[16][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
  const int G = cdiv_dev(*live, group);
  float s = 0.f;
#pragma unroll 4
  for (int k = w; k < G; k += 16) s += dbp[(size_t)k * P + c];   // P is a multiple of 256
  sums[w][lane] = s;
  __syncthreads();
  if (w > 0 || c >= cols) return;
  s = 0.f;
#pragma unroll
  for (int k = 0; k < 16; ++k) s += sums[k][lane];
  db[c] = s * *scal;
}

// dW_s of a piece from the sums over parts of the rows.
__global__ void __launch_bounds__(256) k_vocab_dw(int H, int P, int cols, int S,
                                                  const float* __restrict__ part, VocabOut o) {
  const int c = (blockIdx.x * 256 + threadIdx.x) * 4;
  if (c >= cols) return;
  const int row = blockIdx.y;
  float4 s = f4zero();
  for (int k = 0; k < S; ++k) s = add4(s, ldg4(part + ((size_t)k * H + row) * P + c));
  vocab_store4(o, *o.scale, 0, row, c, s);
}

// dL/dh: live rows from the sums over parts of the vocabulary, the others 0.  A
// workgroup's four wavefronts take a row each, or a quarter of one row's parts
// (WIDE: many parts, few rows), added in their order.  The first workgroup also
// forms the mean loss: a launch less.
template <class OUT, bool WIDE>
__global__ void __launch_bounds__(256) k_vocab_dh(int n, int H, size_t part, int S,
                                                  const int* __restrict__ place,
                                                  const float* __restrict__ sums,
                                                  const float* __restrict__ scal, OUT* dh,
                                                  const float* __restrict__ val,
                                                  const int* __restrict__ live, float* loss) {
  __shared__ float4 quarter[WIDE ? 4 : 1][64];
  if (blockIdx.x == 0 && blockIdx.y == 0) vocab_mean(val, *live, loss);
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int i = WIDE ? blockIdx.x : blockIdx.x * 4 + w, c = (blockIdx.y * 64 + lane) * 4;
  const int per = cdiv_dev(S, 4), z0 = WIDE ? min(w * per, S) : 0, z1 = WIDE ? min(z0 + per, S) : S;
  if (!WIDE && i >= n) return;
  const int k = place[i];
  float4 v = f4zero();
  if (k >= 0 && c < H) {
    const float* p = sums + (size_t)k * H + c;
#pragma unroll 8
    for (int z = z0; z < z1; ++z) v = add4(v, ldg4(p + z * part));
  }
  if constexpr (WIDE) {
    quarter[w][lane] = v;
    __syncthreads();
    if (w > 0) return;
    v = add4(add4(quarter[0][lane], quarter[1][lane]), add4(quarter[2][lane], quarter[3][lane]));
  }
  if (c >= H) return;
  const float x = *scal;
  const float o[4] = {v.x * x, v.y * x, v.z * x, v.w * x};
  store_row<4>(dh + (size_t)i * H + c, o);
}

// Workspace: VocabNet with offsets as its pointers from base.
size_t vocab_net(const cavs_vocab* p, bool train, char* base, VocabNet& v) {
  v = VocabNet{};
  v.n = p->n;
  v.H = p->H;
  v.C = p->C;
  v.K = p->K;
  v.hbf = p->h_type == CAVS_T_BF16;
  v.wbf = v.bf = p->w_type == CAVS_T_BF16;
  // few rows have kernels that read no more of them than there can be
  v.few = p->n <= kVocabFew;
  const int tile = v.few ? kVocabFew : kVocabTile;
  v.rows = (p->n + tile - 1) / tile * tile;
  v.alpha = p->K > 0 ? p->alpha : 0.f;
  v.temp = p->K > 0 ? p->temp : 1.f;
  v.two = p->K > 0 && p->temp != 1.f;
  v.unit = v.alpha < 1.f ? 1.f - v.alpha : v.temp;
  v.distw = v.alpha * v.temp / v.unit;
  v.h = p->h;
  v.bs = p->bs;
  const size_t es = v.bf ? 2 : 4, rows = (size_t)v.rows, H = (size_t)v.H, K = (size_t)v.K;
  size_t o = 0;
  auto take = [&](size_t bytes) {
    const size_t r = o;
    o = align_up(o + bytes, 256);
    return base ? base + r : nullptr;
  };
  v.zrow = (float*)take(256);
  v.live = (int*)take(4);
  v.scal = (float*)take(4);
  v.rows_list = (int*)take(rows * 4);
  v.place = (int*)take(rows * 4);
  v.label = (int*)take(rows * 4);
  v.zlab = (float*)take(rows * 4);
  v.val = (float*)take(rows * 4);
  v.rowc = (float4*)take(rows * 16);
  v.tword = (int*)take(rows * K * 4);
  v.tq = (float*)take(rows * K * 4);
  v.ztop = (float*)take(rows * K * 4);
  v.tsum = (float2*)take(K ? rows * 8 : 0);
  v.slot_words = v.bf ? 128 : 64;
  v.slots = (v.C + v.slot_words - 1) / v.slot_words;
  // the last tile's wavefronts past C have slots too
  const size_t slots = (size_t)((v.C + kVocabTile - 1) / kVocabTile) * (kVocabTile / v.slot_words);
  v.trange = (uint32_t*)take(K ? slots * rows * 4 : 0);
  v.hp = take(rows * H * es);
  // Small tiles where the large ones would leave CUs without one (us, large and
  // small; fp32, fewer than 256 tiles of 128 x 128: 172 x 5 176 x 832 76 and 51, 300
  // x 10 000 x 512 58 and 52, 1000 x 5 000 x 512, 320 tiles, 57 and 66; bf16, fewer
  // than 128 of 256 x 256: 172 x 5 176 x 832 37 and 26, 1000 x 5 000 x 512 31 and 28,
  // 1000 x 10 000 x 1024, 160 tiles, 45 and 70).
  const int big = v.bf ? 256 : 128;
  const long large = (long)((v.n + big - 1) / big) * ((v.C + big - 1) / big);
  v.small = v.few || large < (v.bf ? 128 : 256);
  // The copies straight to LDS want whole 16 bytes of bf16; the small tiles and
  // the fp32 loaders take W_s as it is.
  v.Cq = (v.C + 7) / 8 * 8;
  const bool pad = v.bf && v.Cq != v.C && (train || !v.small);
  v.pad = pad;
  char* wq = take(pad ? H * (size_t)v.Cq * es : 0);
  v.Ws = pad ? wq : p->Ws;
  v.ldw = pad ? v.Cq : v.C;
  const size_t stat = slots * rows * 4;
  v.pm = (float*)take(stat);
  v.ps = (float*)take(stat);
  v.pt = (float*)take(v.two ? stat : 0);
  if (!train) return o;
  // Pieces: dZ of about 256 MB, of equal width, at least 2048 words.  The last
  // ones' tiles are then as full as the first ones'.  In bf16 two of them: the
  // next piece's dz is formed while one is multiplied.
  const size_t words = std::max<size_t>(kPieceBytes / (rows * es), 2048);
  const size_t pieces = ((size_t)v.C + words - 1) / words;
  v.P = (int)(((v.C + pieces - 1) / pieces + kVocabTile - 1) / kVocabTile * kVocabTile);
  v.dz_half = v.bf && v.P < v.C ? rows * v.P * es : 0;
  v.dZ = take(rows * v.P * es + v.dz_half);
  // z is kept, and not formed twice, where it is one piece: in fp32 always (3 ps a
  // value there and back, its product 6 at H = 512); in bf16 while the caches hold
  // it, and from H = 1024 on, where the product takes longer (us with z formed again
  // and kept; 2048 rows, 8 300 words, 68 MB: 126 and 124 at H = 256, 162 and 147 at
  // 512; 3000 rows, 9 000 words, 111 MB: 140 and 156, 184 and 190, at 1024 290 and
  // 270; 4096 rows, 31 000 words: 482 and 552, 718 and 743, 1076 and 1003, at 2048
  // 1914 and 1670).  Few rows always keep it: the tiles that form it again are of
  // 256 rows, their buffers are not.
  const bool keep = v.P >= v.C && (!v.bf || v.few || v.H >= 1024 || rows * v.P * 4 <= kKeepBytes);
  v.Z = keep ? (float*)(v.bf ? take(rows * v.P * 4) : (char*)v.dZ) : nullptr;
  v.keep = keep;
  v.db_rows = 64;
  v.dbp = (float*)take(rows / v.db_rows * v.P * 4);
  // The gradient products split their contraction (Sw, Sh parts, summed
  // afterwards) as far as it shortens the launch; each part costs its way to
  // memory and back.  Times in stages of a tile that has a CU for itself, 1.6 us
  // of either type, or 6.4 MB of traffic.
  const int side = v.bf ? 256 : 128, depth = v.bf ? 64 : 32;
  auto tiles = [&](int x) { return (x + side - 1) / side; };
  auto whole = [](int stages, int S) { return (stages + S - 1) / S; };   // stages of a part
  const int width = std::min(v.P, v.C), tw = tiles(v.H) * tiles(width), th = tiles(v.H) * tiles(v.n);
  const int kw = whole(v.n, depth), kh = whole(width, depth);
  const double wmb = H * (double)v.P * 4e-6, hmb = rows * (double)H * 4e-6;
  auto w_ok = [&](int S) { return S == 1 || (whole(kw, S) >= 4 && S * wmb <= 128); };
  auto h_ok = [&](int S) { return S == 1 || (whole(kh, S) >= 4 && S * hmb <= 64); };
  auto w_cost = [&](int S) { return S > 1 ? 2 * S * wmb / 6.4 + 3 : 0; };
  auto h_cost = [&](int S) { return 2 * S * hmb / 6.4; };
  // One launch, longer items first: it ends about a shorter item after the CUs'
  // mean load, and not before a longer one.  Two fp32 workgroups share a CU: an
  // item takes twice as long beside another, the last ones half of that.  In bf16
  // with pieces the next one's dz follows, in short items; of few rows dL/dh is a
  // launch of its own on small tiles, two a CU.
  const double dz = v.H / 64 + 8., more = v.bf && v.P < v.C ? dz * tiles(v.n) * tiles(width) : 0.;
  const bool apart = v.bf && v.few;
  const double lw = (double)tw * kw / 256, lh = (double)th * kh / 256;
  const double shared = v.bf ? 1. : 2., after = 1. / shared;
  int bw = 1, bh = 1;
  double best = 1e30;
  for (int sw : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64})
    for (int sh : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
      if (!w_ok(sw) || !h_ok(sh)) break;
      const double iw = whole(kw, sw), ih = whole(kh, sh), last = more > 0. ? dz : std::min(iw, ih);
      double t = apart ? std::max(lw, iw) + lh + ih
                       : std::max({lw + lh + more / 256 + after * last, shared * iw, shared * ih});
      t += w_cost(sw) + h_cost(sh);
      if (t < best) best = t, bw = sw, bh = sh;
    }
  v.Sw = whole(kw, whole(kw, bw));   // no part without a stage
  v.Sh = whole(kh, whole(kh, bh));
  v.hpart = (float*)take((size_t)v.Sh * rows * H * 4);
  v.wpart = (float*)take(v.Sw > 1 ? (size_t)v.Sw * H * v.P * 4 : 0);
  return o;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

cavs_status vocab_sizes(cavs_ctx* ctx, const cavs_vocab* p) {
  if (!p) return fail(ctx, CAVS_ERR_ARG, "null vocabulary head");
  if ((p->h_type != CAVS_T_F32 && p->h_type != CAVS_T_BF16) ||
      (p->w_type != CAVS_T_F32 && p->w_type != CAVS_T_BF16))
    return fail(ctx, CAVS_ERR_ARG, "unknown element type");
  if (p->n < 0 || p->H <= 0 || p->C <= 0 || p->K < 0) return fail(ctx, CAVS_ERR_ARG, "bad n/H/C/K");
  if (p->H % 64 != 0) return fail(ctx, CAVS_ERR_UNSUPPORTED, "H=%d not a multiple of 64", p->H);
  if (p->n > kVocabMaxRows || p->C > kVocabMaxWords || p->H > kVocabMaxH)
    return fail(ctx, CAVS_ERR_UNSUPPORTED, "n=%d, C=%d, H=%d: at most %d, %d, %d", p->n, p->C, p->H,
                kVocabMaxRows, kVocabMaxWords, kVocabMaxH);
  if (p->K > kVocabMaxK)
    return fail(ctx, CAVS_ERR_UNSUPPORTED, "K=%d teacher's words (max %d)", p->K, kVocabMaxK);
  if (p->K > 0) {
    if (!(p->alpha >= 0.f && p->alpha <= 1.f)) return fail(ctx, CAVS_ERR_ARG, "alpha outside [0, 1]");
    // T^2 multiplies a difference of sums of a few units, each rounded in 32 bits:
    // past 64 more than some 1e-3 of the loss would be rounding
    if (!(p->temp >= 1.f / 64 && p->temp <= 64.f)) return fail(ctx, CAVS_ERR_ARG, "temp outside [1/64, 64]");
  }
  if (!p->label && p->n > 0 && !(p->K > 0 && p->alpha == 1.f))
    return fail(ctx, CAVS_ERR_ARG, "labels are required unless the teacher alone is learned from");
  return CAVS_OK;
}

cavs_status vocab_args(cavs_ctx* ctx, const cavs_vocab* p) {
  cavs_status st = vocab_sizes(ctx, p);
  if (st != CAVS_OK) return st;
  if (!p->Ws || (p->n > 0 && !p->h)) return fail(ctx, CAVS_ERR_ARG, "h and Ws are required");
  if (!aligned16(p->h) || !aligned16(p->Ws))
    return fail(ctx, CAVS_ERR_ARG, "h and Ws must be aligned to 16 bytes");
  if (p->K > 0 && p->n > 0 && (!p->top_word || !p->top_logit))
    return fail(ctx, CAVS_ERR_ARG, "top_word and top_logit are required with K=%d", p->K);
  return CAVS_OK;
}

template <class IN, class OUT>
void rows(const VocabNet& v, const cavs_vocab* p, float* row_loss, int* err, hipStream_t s) {
  const int R = std::max(16, cdiv(v.n, 4 * 512) * 4);
  CAVS_LAUNCH("k_vocab_rows", (k_vocab_rows<IN, OUT>), dim3(cdiv(v.n, R)), dim3(256), 0, s, v, R, p->label,
              row_loss, err);
}

template <class OUT>
void dh_sum(const VocabNet& v, OUT* dh, float* loss, hipStream_t s) {
  const size_t part = (size_t)v.rows * v.H;
  const int gx = cdiv(v.H, 256);
  if (v.Sh >= 8)
    CAVS_LAUNCH("k_vocab_dh", (k_vocab_dh<OUT, true>), dim3(v.n, gx), dim3(256), 0, s, v.n, v.H, part, v.Sh,
                v.place, v.hpart, v.scal, dh, v.val, v.live, loss);
  else
    CAVS_LAUNCH("k_vocab_dh", (k_vocab_dh<OUT, false>), dim3(cdiv(v.n, 4), gx), dim3(256), 0, s, v.n, v.H, part,
                v.Sh, v.place, v.hpart, v.scal, dh, v.val, v.live, loss);
}

}  // namespace

VocabEp vocab_ep(const VocabNet& v, int col0) {
  return VocabEp{v.C,   col0,   v.K,  v.rows, v.two,  1.f / v.temp, v.distw, v.live,
                 v.bs,  v.label, v.tword, v.tq, v.trange, v.pm, v.ps, v.pt, v.zlab, v.ztop, v.Z, v.rowc,
                 v.P > 0 ? vocab_dz_at(v, col0) : nullptr, v.P, v.dbp};
}

size_t vocab_ws_bytes(const cavs_vocab* p, bool train) {
  if (vocab_sizes(nullptr, p) != CAVS_OK) return 0;
  VocabNet v;
  return p->n > 0 ? vocab_net(p, train, nullptr, v) : 0;
}

cavs_status vocab_run(cavs_ctx* ctx, const cavs_vocab* p, float* loss, float* row_loss, void* dh,
                      void* dWs, float* dbs, void* ws, size_t ws_bytes, bool train) {
  cavs_status st = vocab_args(ctx, p);
  if (st != CAVS_OK) return st;
  if (!loss) return fail(ctx, CAVS_ERR_ARG, "loss is required");
  if (train) {
    if (!dWs || (p->n > 0 && !dh)) return fail(ctx, CAVS_ERR_ARG, "dh and dWs are required");
    if ((p->bs != nullptr) != (dbs != nullptr))
      return fail(ctx, CAVS_ERR_ARG, "dbs goes with bs");
    if (!aligned16(dh) || !aligned16(dWs))
      return fail(ctx, CAVS_ERR_ARG, "dh and dWs must be aligned to 16 bytes");
  }
  hipStream_t s = ctx->stream;
  if (p->n == 0) {
    CAVS_HIP_CHECK(ctx, zero_async(loss, 4, s));
    if (train) {
      const size_t e = (size_t)p->H * p->C;
      CAVS_HIP_CHECK(ctx, zero_async(dWs, e * (p->w_type == CAVS_T_BF16 ? 2 : 4), s));
      if (dbs) CAVS_HIP_CHECK(ctx, zero_async(dbs, (size_t)p->C * 4, s));
    }
    return CAVS_OK;
  }
  VocabNet v;
  const size_t need = vocab_net(p, train, (char*)ws, v);
  if (!ws || ws_bytes < need)
    return fail(ctx, CAVS_ERR_WORKSPACE, "workspace too small: %zu < %zu", ws_bytes, need);
  if (!aligned16(ws)) return fail(ctx, CAVS_ERR_ARG, "ws must be aligned to 16 bytes");

  int* err = ctx->dev_err_dev;
  if (v.hbf) v.bf ? rows<u16, u16>(v, p, row_loss, err, s) : rows<u16, float>(v, p, row_loss, err, s);
  else v.bf ? rows<float, u16>(v, p, row_loss, err, s) : rows<float, float>(v, p, row_loss, err, s);
  if (v.pad)
    CAVS_LAUNCH("k_vocab_pad", k_vocab_pad, dim3(cdiv(v.C, 256 * 8), v.H), dim3(256), 0, s, v.H, v.C, v.Cq,
                (const u16*)p->Ws, (u16*)v.Ws);
  if (v.K > 0)
    CAVS_LAUNCH("k_vocab_teacher", k_vocab_teacher, dim3(v.rows / 4), dim3(256), 0, s, v, p->top_word,
                p->top_logit, err);
  v.bf ? vocab_bf_loss(v, p->Ws, s) : vocab_x3_loss(v, p->Ws, s);
  // the mean: with the gradients in their last kernel, else here or by itself
  const bool one = !train && v.n <= 16;
  CAVS_LAUNCH("k_vocab_join", k_vocab_join, dim3(one ? 1 : v.rows / 16), dim3(1024), 0, s, v, row_loss,
              one ? loss : nullptr);
  if (!train && !one)
    CAVS_LAUNCH("k_vocab_mean", k_vocab_mean, dim3(1), dim3(256), 0, s, v.val, v.live, loss);
  if (train) {
    auto width = [&](int col0) { return std::max(0, std::min(v.P, v.C - col0)); };
    auto db = [&](int col0) {
      if (dbs)
        CAVS_LAUNCH("k_vocab_db", k_vocab_db, dim3(cdiv(width(col0), 64)), dim3(1024), 0, s, width(col0), v.P,
                    v.db_rows, v.live, v.dbp, v.scal, dbs + col0);
    };
    for (int col0 = 0; col0 < v.C; col0 += v.P) {
      const int cols = width(col0), next = width(col0 + v.P);
      if (v.keep) {
        const dim3 grid(v.P / 256, v.rows / 64);
        float* const all = v.rows == v.db_rows ? dbs : nullptr;
        if (v.bf) CAVS_LAUNCH("k_vocab_dz", k_vocab_dz<u16>, grid, dim3(256), 0, s, v, all);
        else CAVS_LAUNCH("k_vocab_dz", k_vocab_dz<float>, grid, dim3(256), 0, s, v, all);
      } else if (!v.bf) {
        vocab_x3_dz(v, col0, cols, s);
      } else if (col0 == 0) {
        vocab_bf_dz(v, col0, cols, s);
      }
      if ((!v.bf || col0 == 0) && !(v.keep && v.rows == v.db_rows)) db(col0);
      char* at = (char*)dWs + (size_t)col0 * (v.wbf ? 2 : 4);
      const VocabOut out{at, v.C, 0, v.H, cols, v.wbf, 0, v.scal};
      const VocabOut sums{v.wpart, v.P, (size_t)v.H * v.P, v.H, cols, 0, 0, nullptr};
      const VocabOut& o = v.Sw > 1 ? sums : out;
      if (v.bf) {
        vocab_bf_grads(v, col0, cols, next, o, s);
        if (next > 0) db(col0 + v.P);
      } else {
        vocab_x3_grads(v, col0, cols, o, s);
      }
      if (v.Sw > 1)
        CAVS_LAUNCH("k_vocab_dw", k_vocab_dw, dim3(cdiv(cols, 1024), v.H), dim3(256), 0, s, v.H, v.P, cols,
                    v.Sw, v.wpart, out);
    }
    v.hbf ? dh_sum(v, (u16*)dh, loss, s) : dh_sum(v, (float*)dh, loss, s);
  }
  CAVS_LAUNCH_CHECK(ctx);
  return CAVS_OK;
}

}  // namespace cavs
