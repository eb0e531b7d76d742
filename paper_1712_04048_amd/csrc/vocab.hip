// The vocabulary head: the live rows, the teacher's distributions, the
// softmax statistics joined over the vocabulary, the loss, and the order of the
// products (vocab_x3.hip, vocab_bf.hip).
//
//   loss       z = h W_s + b_s tile by tile; a tile leaves each row's largest z
//              and sum of exponentials over its words, never z itself
//   gradient   for each piece of P words: z again, dz from the joined
//              statistics into dZ [rows, P], then dW_s of the piece = h^T dZ and
//              dL/dh += dZ W_s^T
// The second pass over z costs two of eight units of work; what it saves is
// rows x C values of memory (the head inside cavs_forward keeps them).
#include <math.h>

#include <algorithm>

#include "vocab.h"

namespace cavs {
namespace {

// Sizes whose tiles and offsets the kernels count in 32 bits.
constexpr int kVocabMaxRows = 1 << 20, kVocabMaxWords = 1 << 20, kVocabMaxH = 1 << 15;

// Live rows in ascending order, their labels, unit / their number.  One
// workgroup: 8192 rows are eight rounds.
__global__ void __launch_bounds__(1024) k_vocab_rows(int n, int C, const int* __restrict__ label,
                                                     int* rows, int* place, int* clabel, int* live, float unit,
                                                     float* scal,
                                                     float* row_loss, float* zrow, int* err) {
  __shared__ int wsum[16];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  if (tid < 64) zrow[tid] = 0.f;
  int done = 0;
  bool bad = false;
  for (int base = 0; base < n; base += 1024) {
    const int i = base + tid;
    const int y = i < n ? (label ? label[i] : 0) : -1;
    bad |= y < -1 || y >= C;
    const bool on = y >= 0 && y < C;
    const unsigned long long m = __ballot(on);
    if (lane == 0) wsum[w] = __popcll(m);
    __syncthreads();
    int before = done, total = 0;
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      if (k < w) before += wsum[k];
      total += wsum[k];
    }
    if (on) {
      const int at = before + __popcll(m & ((1ull << lane) - 1));
      rows[at] = i;
      clabel[at] = label ? y : -1;
      place[i] = at;
    } else if (i < n) {
      place[i] = -1;
      if (row_loss) row_loss[i] = 0.f;
    }
    done += total;
    __syncthreads();
  }
  if (bad) err[1] = 1;
  if (tid == 0) {
    *live = done;
    scal[0] = unit / (float)max(done, 1);
  }
}

// The live rows of h in the products' type, zeros to the end of their tile.
template <class IN, class OUT>
__global__ void __launch_bounds__(256) k_vocab_pack(int H, const IN* __restrict__ h,
                                                    const int* __restrict__ rows,
                                                    const int* __restrict__ live, OUT* hp) {
  const int nl = *live, end = (nl + kVocabTile - 1) / kVocabTile * kVocabTile;
  const int q = H / 4;   // H is a multiple of 64
  for (int row = blockIdx.x * 4 + (threadIdx.x >> 6); row < end; row += gridDim.x * 4) {
    const IN* src = row < nl ? h + (size_t)rows[row] * H : nullptr;
    OUT* dst = hp + (size_t)row * H;
    for (int c = threadIdx.x & 63; c < q; c += 64) {
      float4 v = f4zero();
      if (src) {
        if constexpr (sizeof(IN) == 4) {
          v = ldg4((const float*)src + 4 * c);
        } else {
          const uint2 x = *reinterpret_cast<const uint2*>(src + 4 * c);
          v = make_float4(__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xffff0000u),
                          __uint_as_float(x.y << 16), __uint_as_float(x.y & 0xffff0000u));
        }
      }
      if constexpr (sizeof(OUT) == 4) st4((float*)dst + 4 * c, v);
      else st_bf4((u16*)dst + 4 * c, v);
    }
  }
}

// W_s with its rows padded to whole 16 bytes (zeros), for a C that is not.
template <class T>
__global__ void __launch_bounds__(256) k_vocab_pad(int C, int Cq, const T* __restrict__ W, T* out) {
  const size_t row = blockIdx.y;
  for (int c = blockIdx.x * 256 + threadIdx.x; c < Cq; c += gridDim.x * 256)
    out[row * Cq + c] = c < C ? W[row * C + c] : T(0);
}

// The teacher's distribution over its words of a live row: q = softmax(t / T)
// over the words that are there and have a logit above -inf.  A word that is
// listed twice counts as the sum of its entries, at its first place, so that
// the products' epilogues change each word once; the loss's sum of q ln q is
// over the entries.  A wavefront per row; K at most kVocabMaxK.
__global__ void __launch_bounds__(256) k_vocab_teacher(int C, int K, float invT,
                                                       const int* __restrict__ rows,
                                                       const int* __restrict__ live,
                                                       const int* __restrict__ top_word,
                                                       const float* __restrict__ top_logit,
                                                       int* tword, float* tq, float2* tsum, int* err) {
  constexpr int PER = kVocabMaxK / 64;
  __shared__ int words[4][kVocabMaxK];
  __shared__ float qs[4][kVocabMaxK];
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63, row = blockIdx.x * 4 + w;
  const int nl = *live;
  if (row < nl) {
    const size_t src = (size_t)rows[row] * K;
    int id[PER];
    float t[PER], m = -INFINITY;
    bool bad = false;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int j = lane + 64 * k;
      id[k] = j < K ? top_word[src + j] : -1;
      bad |= id[k] < -1 || id[k] >= C;
      if (id[k] >= C) id[k] = -1;
      t[k] = id[k] >= 0 ? top_logit[src + j] * invT : -INFINITY;
      m = fmaxf(m, t[k]);
    }
    if (bad) err[1] = 1;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, kWave));
    // nothing there: all -inf (a NaN among them is not nothing)
    bool nan = false;
#pragma unroll
    for (int k = 0; k < PER; ++k) nan |= t[k] != t[k];
    const bool some = m > -INFINITY || __any(nan);
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
    if (lane == 0) tsum[row] = make_float2(s, some ? 1.f : 0.f);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int j = lane + 64 * k;
      if (j >= K) continue;
      bool first = true;
      float total = 0.f;
      for (int i = 0; i < K; ++i) {
        const bool same = words[w][i] == id[k];
        first = first && !(same && i < j);
        total += same ? qs[w][i] : 0.f;
      }
      const size_t at = (size_t)row * K + j;
      tword[at] = first ? id[k] : -1;
      tq[at] = total;
    }
  }
}

// A row's statistics joined over the slots, its loss, and what its dz is made
// from.  64 rows a workgroup, sixteen wavefronts on every sixteenth slot each,
// their sums added in their order.
//   CE = ln(sum exp(z - m)) + m - z_label
//   KD = T^2 (sum q ln q + ln(sum exp((z - m) / T)) + sum q (m - z) / T)
__global__ void __launch_bounds__(1024) k_vocab_join(VocabNet v, float* row_loss) {
  __shared__ float sm[16][64], ss[16][64], st[16][64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, row = blockIdx.x * 64 + lane;
  const int nl = *v.live;
  if ((int)blockIdx.x * 64 >= nl) {
    // the rest of the last tile of 256 rows
    if (w == 0 && (int)blockIdx.x * 64 < cdiv_dev(nl, kVocabTile) * kVocabTile)
      v.rowc[row] = f4zero();
    return;
  }
  float m = -INFINITY;
  for (int k = w; k < v.slots; k += 16) m = fmaxf(m, v.pm[(size_t)k * v.rows + row]);
  sm[w][lane] = m;
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 16; ++k) m = fmaxf(m, sm[k][lane]);
  const float mm = m == -INFINITY ? 0.f : m;
  float s = 0.f, t = 0.f;
  for (int k = w; k < v.slots; k += 16) {
    const size_t at = (size_t)k * v.rows + row;
    const float d = (v.pm[at] - mm) * kLog2e;
    s += v.ps[at] * __builtin_amdgcn_exp2f(d);
    if (v.two) t += v.pt[at] * __builtin_amdgcn_exp2f(d / v.temp);
  }
  ss[w][lane] = s;
  st[w][lane] = t;
  __syncthreads();
  if (w > 0) return;
  s = 0.f;
  t = 0.f;
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    s += ss[k][lane];
    t += st[k][lane];
  }
  if (!v.two) t = s;
  if (row >= nl) {
    v.rowc[row] = f4zero();
    return;
  }
  float val = 0.f, has = 0.f;
  const float a = v.K > 0 ? v.alpha : 0.f;
  const int y = v.label[row];
  if (y >= 0 && a < 1.f) val = (1.f - a) * (logf(s) + (m - v.zlab[row]));
  if (v.K > 0) {
    const float2 q = v.tsum[row];
    has = q.y;
    if (has != 0.f && a > 0.f) {
      float dot = 0.f;
      for (int j = 0; j < v.K; ++j) {
        const size_t at = (size_t)row * v.K + j;
        const float p = v.tq[at];
        if (v.tword[at] >= 0 && p != 0.f) dot += p * (m - v.ztop[at]);
      }
      val += a * v.temp * v.temp * (q.x + logf(t) + dot / v.temp);
    }
  }
  v.val[row] = val;
  if (row_loss) row_loss[v.rows_list[row]] = val;
  // in units of v.unit
  const float lab = a < 1.f ? 1.f : 0.f, c1 = lab != 0.f ? 1.f / s : 0.f;
  const float cT = has != 0.f ? v.distw / t : 0.f;
  v.rowc[row] = v.two ? make_float4(m, c1, cT, lab) : make_float4(m, c1 + cT, 0.f, lab);
}

// The mean of the live rows' losses, in 64 bits and a fixed order.
__global__ void __launch_bounds__(1024) k_vocab_mean(const float* __restrict__ val,
                                                     const int* __restrict__ live, float* loss) {
  __shared__ double part[16];
  const int nl = *live;
  double s = 0.0;
  for (int i = threadIdx.x; i < nl; i += 1024) s += (double)val[i];
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o, kWave);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0;
    for (int k = 0; k < 16; ++k) s += part[k];
    *loss = (float)(s / (double)max(nl, 1));
  }
}

// db_s of a piece: the groups' sums in order.
__global__ void __launch_bounds__(256) k_vocab_db(int cols, int P, int group,
                                                  const int* __restrict__ live,
                                                  const float* __restrict__ dbp,
                                                  const float* __restrict__ scal, float* db) {
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= cols) return;
  const int G = cdiv_dev(*live, group);
  float s = 0.f;
  for (int k = 0; k < G; ++k) s += dbp[(size_t)k * P + c];
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

// dL/dh: live rows from the sums over parts of the vocabulary, the others 0.
template <class OUT>
__global__ void __launch_bounds__(256) k_vocab_dh(int n, int H, size_t part, int S,
                                                  const int* __restrict__ place,
                                                  const float* __restrict__ sums,
                                                  const float* __restrict__ scal, OUT* dh) {
  const int q = H / 4, lane = threadIdx.x & 63;
  const float w = *scal;
  for (int i = blockIdx.x * 4 + (threadIdx.x >> 6); i < n; i += gridDim.x * 4) {
    const int k = place[i];
    for (int c = lane; c < q; c += 64) {
      float4 v = f4zero();
      if (k >= 0)
        for (int z = 0; z < S; ++z) v = add4(v, ldg4(sums + z * part + (size_t)k * H + 4 * c));
      v = make_float4(v.x * w, v.y * w, v.z * w, v.w * w);
      if constexpr (sizeof(OUT) == 4) st4((float*)dh + (size_t)i * H + 4 * c, v);
      else st_bf4((u16*)dh + (size_t)i * H + 4 * c, v);
    }
  }
}

// Workspace: VocabNet with offsets as its pointers from base.
size_t vocab_net(const cavs_vocab* p, bool train, char* base, VocabNet& v) {
  v = VocabNet{};
  v.n = p->n;
  v.H = p->H;
  v.C = p->C;
  v.K = p->K;
  v.rows = (p->n + kVocabTile - 1) / kVocabTile * kVocabTile;
  v.hbf = p->h_type == CAVS_T_BF16;
  v.wbf = v.bf = p->w_type == CAVS_T_BF16;
  v.alpha = p->K > 0 ? p->alpha : 0.f;
  v.temp = p->K > 0 ? p->temp : 1.f;
  v.two = p->K > 0 && p->temp != 1.f;
  v.unit = v.alpha < 1.f ? 1.f - v.alpha : v.temp;
  v.distw = v.alpha * v.temp / v.unit;
  v.h = p->h;
  v.bs = p->bs;
  const size_t es = v.bf ? 2 : 4, rows = (size_t)v.rows, H = (size_t)v.H, K = (size_t)v.K;
  const int vec = (int)(16 / es);
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
  v.hp = take(rows * H * es);
  v.Cq = (v.C + vec - 1) / vec * vec;
  const bool pad = v.Cq != v.C;
  char* wq = take(pad ? H * (size_t)v.Cq * es : 0);
  v.Ws = pad ? wq : p->Ws;
  v.ldw = v.Cq;
  v.slot_words = v.bf ? 128 : 64;
  v.slots = (v.C + v.slot_words - 1) / v.slot_words;
  // a slot more than joined: the last tile's wavefronts past C write theirs
  const size_t stat = (size_t)((v.C + kVocabTile - 1) / kVocabTile) * (kVocabTile / v.slot_words) * rows * 4;
  v.pm = (float*)take(stat);
  v.ps = (float*)take(stat);
  v.pt = (float*)take(v.two ? stat : 0);
  if (!train) return o;
  // Pieces: dZ of about 256 MB, of equal width, at least 2048 words.  The last
  // ones' tiles are then as full as the first ones'.
  const size_t words = std::max<size_t>(((size_t)256 << 20) / (rows * es), 2048);
  const size_t pieces = ((size_t)v.C + words - 1) / words;
  v.P = (int)(((v.C + pieces - 1) / pieces + kVocabTile - 1) / kVocabTile * kVocabTile);
  v.dZ = take(rows * v.P * es);
  v.db_rows = 64;
  v.dbp = (float*)take(rows / v.db_rows * v.P * 4);
  // The gradient products are split over their contraction until a workgroup
  // per CU is there, each part at least four stages deep and the parts of dh
  // at most 64 MB (dW's: 128).
  const int tile = v.bf ? 256 : 128, depth = v.bf ? 64 : 32, want = v.bf ? 256 : 512;
  auto parts = [&](int tiles, int stages, size_t bytes, size_t cap) {
    int S = std::max(1, std::min({want / std::max(tiles, 1), stages / 4,
                                  (int)std::min<size_t>(cap / std::max<size_t>(bytes, 1), 64)}));
    return (stages + (stages + S - 1) / S - 1) / ((stages + S - 1) / S);   // no part without a stage
  };
  auto tiles = [&](int x) { return (x + tile - 1) / tile; };
  const int width = std::min(v.P, v.C);
  v.Sh = parts(tiles(v.H) * tiles(v.n), (width + depth - 1) / depth, rows * H * 4, (size_t)64 << 20);
  v.hpart = (float*)take((size_t)v.Sh * rows * H * 4);
  v.Sw = parts(tiles(v.H) * tiles(width), v.rows / depth, H * v.P * 4, (size_t)128 << 20);
  v.wpart = (float*)take(v.Sw > 1 ? (size_t)v.Sw * H * v.P * 4 : 0);
  return o;
}

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

cavs_status vocab_args(cavs_ctx* ctx, const cavs_vocab* p) {
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
  if (!p->Ws || (p->n > 0 && !p->h)) return fail(ctx, CAVS_ERR_ARG, "h and Ws are required");
  if (!aligned16(p->h) || !aligned16(p->Ws))
    return fail(ctx, CAVS_ERR_ARG, "h and Ws must be aligned to 16 bytes");
  if (p->K > 0) {
    if (p->n > 0 && (!p->top_word || !p->top_logit))
      return fail(ctx, CAVS_ERR_ARG, "top_word and top_logit are required with K=%d", p->K);
    if (!(p->alpha >= 0.f && p->alpha <= 1.f)) return fail(ctx, CAVS_ERR_ARG, "alpha outside [0, 1]");
    if (!(p->temp > 0.f && p->temp < INFINITY)) return fail(ctx, CAVS_ERR_ARG, "temp must be positive");
  }
  if (!p->label && p->n > 0 && !(p->K > 0 && p->alpha == 1.f))
    return fail(ctx, CAVS_ERR_ARG, "labels are required unless the teacher alone is learned from");
  return CAVS_OK;
}

template <class IN, class OUT>
void pack(const VocabNet& v, hipStream_t s) {
  CAVS_LAUNCH("k_vocab_pack", (k_vocab_pack<IN, OUT>), dim3(std::min(v.rows / 4, 8192)), dim3(256), 0, s,
              v.H, (const IN*)v.h, v.rows_list, v.live, (OUT*)v.hp);
}

}  // namespace

VocabEp vocab_ep(const VocabNet& v, int col0) {
  return VocabEp{v.C,   col0,   v.K,  v.rows, v.two,  1.f / v.temp, v.distw, v.live,
                 v.bs,  v.label, v.tword, v.tq, v.pm, v.ps, v.pt, v.zlab, v.ztop, v.rowc,
                 v.dZ,  v.P,  v.dbp};
}

size_t vocab_ws_bytes(const cavs_vocab* p, bool train) {
  if (vocab_args(nullptr, p) != CAVS_OK) return 0;
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
  const size_t need = vocab_net(p, train, nullptr, v);
  if (!ws || ws_bytes < need)
    return fail(ctx, CAVS_ERR_WORKSPACE, "workspace too small: %zu < %zu", ws_bytes, need);
  if (!aligned16(ws)) return fail(ctx, CAVS_ERR_ARG, "ws must be aligned to 16 bytes");
  vocab_net(p, train, (char*)ws, v);

  CAVS_LAUNCH("k_vocab_rows", k_vocab_rows, dim3(1), dim3(1024), 0, s, v.n, v.C, p->label, v.rows_list,
              v.place, v.label, v.live, v.unit, v.scal, row_loss, v.zrow, ctx->dev_err_dev);
  if (v.hbf) v.bf ? pack<u16, u16>(v, s) : pack<u16, float>(v, s);
  else v.bf ? pack<float, u16>(v, s) : pack<float, float>(v, s);
  if (v.Cq != v.C) {
    const dim3 grid(std::min(cdiv(v.Cq, 256), 64), v.H);
    if (v.bf)
      CAVS_LAUNCH("k_vocab_pad", k_vocab_pad<u16>, grid, dim3(256), 0, s, v.C, v.Cq, (const u16*)p->Ws,
                  (u16*)v.Ws);
    else
      CAVS_LAUNCH("k_vocab_pad", k_vocab_pad<float>, grid, dim3(256), 0, s, v.C, v.Cq,
                  (const float*)p->Ws, (float*)v.Ws);
  }
  if (v.K > 0)
    CAVS_LAUNCH("k_vocab_teacher", k_vocab_teacher, dim3(v.rows / 4), dim3(256), 0, s, v.C, v.K,
                1.f / v.temp, v.rows_list, v.live, p->top_word, p->top_logit, v.tword, v.tq, v.tsum,
                ctx->dev_err_dev);
  v.bf ? vocab_bf_loss(v, s) : vocab_x3_loss(v, s);
  CAVS_LAUNCH("k_vocab_join", k_vocab_join, dim3(v.rows / 64), dim3(1024), 0, s, v, row_loss);
  CAVS_LAUNCH("k_vocab_mean", k_vocab_mean, dim3(1), dim3(1024), 0, s, v.val, v.live, loss);
  if (train) {
    for (int col0 = 0; col0 < v.C; col0 += v.P) {
      const int cols = std::min(v.P, v.C - col0);
      v.bf ? vocab_bf_dz(v, col0, cols, s) : vocab_x3_dz(v, col0, cols, s);
      if (dbs)
        CAVS_LAUNCH("k_vocab_db", k_vocab_db, dim3(cdiv(cols, 256)), dim3(256), 0, s, cols, v.P,
                    v.db_rows, v.live, v.dbp, v.scal, dbs + col0);
      char* at = (char*)dWs + (size_t)col0 * (v.wbf ? 2 : 4);
      const VocabOut out{at, v.C, 0, v.H, cols, v.wbf, 0, v.scal};
      const VocabOut sums{v.wpart, v.P, (size_t)v.H * v.P, v.H, cols, 0, 0, nullptr};
      const VocabOut& o = v.Sw > 1 ? sums : out;
      v.bf ? vocab_bf_dw(v, col0, cols, o, s) : vocab_x3_dw(v, col0, cols, o, s);
      if (v.Sw > 1)
        CAVS_LAUNCH("k_vocab_dw", k_vocab_dw, dim3(cdiv(cols, 1024), v.H), dim3(256), 0, s, v.H, v.P, cols,
                    v.Sw, v.wpart, out);
      v.bf ? vocab_bf_dh(v, col0, cols, s) : vocab_x3_dh(v, col0, cols, s);
    }
    const dim3 grid(std::min(cdiv(v.n, 4), 8192));
    if (v.hbf)
      CAVS_LAUNCH("k_vocab_dh", k_vocab_dh<u16>, grid, dim3(256), 0, s, v.n, v.H, (size_t)v.rows * v.H, v.Sh,
                  v.place, v.hpart, v.scal, (u16*)dh);
    else
      CAVS_LAUNCH("k_vocab_dh", k_vocab_dh<float>, grid, dim3(256), 0, s, v.n, v.H, (size_t)v.rows * v.H,
                  v.Sh, v.place, v.hpart, v.scal, (float*)dh);
  }
  CAVS_LAUNCH_CHECK(ctx);
  return CAVS_OK;
}

}  // namespace cavs
