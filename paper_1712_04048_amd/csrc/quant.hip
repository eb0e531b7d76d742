// A head in 4 bits: its rounding, and its product with a few rows.
//
//   What[k, c] = s[g, c] (q[k, c] - 8) + m[g, c],  g = k / group,  q in 0 .. 15
//
// Layout.  Words are cut into tiles of 16, rows of W into blocks of 128; a tile's
// block is 1024 bytes, 16 for each lane l = 16 j + (c % 16) of a wavefront: four
// dwords, dword b holding k = 32 b + 8 j + i, i = 0 .. 7, of column c -- what the
// lane feeds to the four 32-deep matrix instructions of the block.  Nibble p of a
// dword (bits 4p ..) is i = 2p (p < 4) or 2 (p - 4) + 1: two masks and a shift then
// leave adjacent i in the two halves of a register.  A tile's blocks follow each
// other, then the next tile's.  The scales come after all codes: for each tile,
// block and column the 128 / group scales of its groups (bf16), each followed by its
// shift where there are any.  What is past H or C has q = 8 and s = m = 0.
#include <algorithm>

#include "vocab.h"
#include "xcd_map.h"

namespace cavs {
namespace {

constexpr int kQuantMaxH = 1 << 15, kQuantMaxC = 1 << 20, kQuantMaxN = 1 << 20;
constexpr int kQB = 128;   // rows of W in a block
constexpr int kQR = 16;    // rows of x of a workgroup, at most
constexpr int kQW = 16;    // wavefronts of a workgroup
constexpr size_t kQLds = 152 << 10;   // most LDS of a workgroup

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

struct QuantNet {
  int H, C, T, KB;             // T tiles of 16 words, KB blocks of kQB rows
  const uint4* code;           // [T][KB][64]
  const u16* scale;            // [T][KB][16][128 / group][1 + shift]
};

__device__ __forceinline__ float load_one(const float* p) { return *p; }
__device__ __forceinline__ float load_one(const u16* p) { return __uint_as_float((uint32_t)*p << 16); }
__device__ __forceinline__ void store_one(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_one(u16* p, float v) { *p = f2bf(v); }
__device__ __forceinline__ float bf2f(u16 v) { return __uint_as_float((uint32_t)v << 16); }

// To fp32 and then to bf16, as the format says; in one expression with contraction
// the two roundings become one.
__device__ __forceinline__ u16 round_twice(double v) {
#pragma clang fp contract(off)
  const float f = (float)v;
  return f2bf(f);
}

// The whole number nearest to (w - m) / s, the even one of two, in -8 .. 7, by the
// definition: where fp32 does not hold 1 / s, or what is multiplied with it.
__device__ __noinline__ float quant_code_wide(float w, float s, float m) {
  return fminf(fmaxf((float)rint(((double)w - (double)m) / (double)s), -8.f), 7.f);
}

// The same for a scale well inside fp32's range, inv = 1 / s.  d = w - m is rounded
// once, which leaves it on its side of each border b s (b half way between two codes):
// b s is a float of at most 13 bits.  t2 is d / s rounded once (a quotient within two
// steps of it, corrected by its own remainder, which the fused product has exactly);
// a float d other than b s is at least 2^-23 / (its mantissa) of b s away from it, more
// than half a step of t2 at b, so t2 is b for d = b s alone.  With m = 0 d is w and
// the even one is right; with a shift d may have been rounded to b s, and w - m, which
// 64 bits hold, decides.
template <bool SHIFT>
__device__ __forceinline__ float quant_code(float w, float s, float m, float inv) {
  const float d = SHIFT ? w - m : w, t = d * inv, t2 = fmaf(fmaf(-t, s, d), inv, t);
  float q = rintf(t2);
  if (SHIFT && fabsf(t2 - q) == 0.5f) {
    const double over = fma(-(double)t2, (double)s, (double)w - (double)m);
    if (over != 0.0) q = (over > 0.0) == (s > 0.f) ? t2 + 0.5f : t2 - 0.5f;
  }
  return __builtin_amdgcn_fmed3f(q, -8.f, 7.f);
}

// Eight codes plus 8 in the order of a dword: the even places are nibbles 0 .. 3, the
// odd ones 4 .. 7, summed as floats, which hold four of them; 8 in each is 0x8888.
template <bool SHIFT>
__device__ __forceinline__ uint32_t quant_codes(const float (&w)[8], float s, float m, float inv) {
  float q[8];
  if (fabsf(s) > 0x1p-100f && fabsf(s) < 0x1p100f) {
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = quant_code<SHIFT>(w[i], s, m, inv);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = quant_code_wide(w[i], s, m);
  }
  const float even = fmaf(fmaf(fmaf(q[6], 16.f, q[4]), 16.f, q[2]), 16.f, q[0]) + 34952.f;
  const float odd = fmaf(fmaf(fmaf(q[7], 16.f, q[5]), 16.f, q[3]), 16.f, q[1]) + 34952.f;
  return (uint32_t)even | (uint32_t)odd << 16;
}

// 64 columns of a block of 128 rows to a workgroup, sixteen rows to a wavefront, in
// registers, so that W is read once; a group's ends are joined through LDS, and the
// dwords are put into the layout's order there.  Bound by memory: W once in, 4 bits a
// weight out.  Each XCD takes adjacent columns: rows of any length then share the
// lines at a workgroup's ends in its cache (1024 x 50 001: bf16 with shifts 42 us with
// neighbours on other XCDs and 35 here, 3.8 TB/s; fp32 86 and 71).  Two or four
// columns a lane were no faster (38 and 48).
template <class T, int G, bool SHIFT>
__global__ void __launch_bounds__(512) k_quant_pack(QuantNet q, const T* __restrict__ W, uint4* code, u16* scale) {
  constexpr int GW = G / 16;   // wavefronts of a group
  __shared__ float ends[2][8][64];
  __shared__ uint32_t dw[4][4][4][16];   // [b][tile][j][column]
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nx = cdiv_dev(q.C, 64), item = xcd_item(blockIdx.x, nx * q.KB);
  if (item < 0) return;
  const int kb = item / nx, bx = item - kb * nx, c = bx * 64 + lane, k0 = kb * kQB + 16 * w;
  const int rows = min(16, q.H - k0);   // may be negative
  const bool in = c < q.C;
  // past the last row it again, which changes no group's ends
  float x[16];
  if (in) {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = load_one(W + (size_t)min(k0 + i, q.H - 1) * q.C + c);
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = 0.f;
  }
  float lo = INFINITY, hi = -INFINITY, odd = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    lo = fminf(lo, x[i]);
    hi = fmaxf(hi, x[i]);
    odd = fmaf(x[i], 0.f, odd);   // NaN where one is not finite
  }
  ends[0][w][lane] = odd == 0.f ? lo : -INFINITY;
  ends[1][w][lane] = odd == 0.f ? hi : INFINITY;
  __syncthreads();
  const int w0 = w & ~(GW - 1), tile = bx * 4 + lane / 16;
#pragma unroll
  for (int i = 0; i < GW; ++i) {
    lo = fminf(lo, ends[0][w0 + i][lane]);
    hi = fmaxf(hi, ends[1][w0 + i][lane]);
  }
  u16 s16 = 0, m16 = 0;
  if (in && kb * kQB + 16 * w0 < q.H) {   // the group has rows
    if (hi == INFINITY) {
      s16 = 0x7fc0;
    } else if (SHIFT) {
      s16 = round_twice(((double)hi - (double)lo) / 15.0);
      m16 = round_twice(0.5 * ((double)lo + (double)hi) + 0.5 * (double)bf2f(s16));
    } else {
      // the end that is further from 0 (the lower of two alike) becomes -8
      s16 = f2bf(-0.125f * (hi > -lo ? hi : lo));
    }
  }
  const float s = bf2f(s16), m = SHIFT ? bf2f(m16) : 0.f, inv = 1.f / s;
  if (rows < 16)
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = i < rows ? x[i] : m;
#pragma unroll
  for (int jj = 0; jj < 2; ++jj) {
    float v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = x[8 * jj + i];
    dw[w / 2][lane / 16][w % 2 * 2 + jj][lane % 16] =
        s != 0.f && s == s ? quant_codes<SHIFT>(v, s, m, inv) : 0x88888888u;
  }
  if (tile < q.T && w == w0) {
    constexpr int W16 = kQB / G * (SHIFT ? 2 : 1);
    u16* at = scale + (((size_t)tile * q.KB + kb) * 16 + lane % 16) * W16 + w / GW * (SHIFT ? 2 : 1);
    at[0] = s16;
    if (SHIFT) at[1] = m16;
  }
  __syncthreads();
  const int t = threadIdx.x / 64;
  if (t < 4 && bx * 4 + t < q.T)
    code[((size_t)(bx * 4 + t) * q.KB + kb) * 64 + lane] =
        make_uint4((&dw[0][t][0][0])[lane], (&dw[1][t][0][0])[lane], (&dw[2][t][0][0])[lane], (&dw[3][t][0][0])[lane]);
}

// What in rows, a dword of eight rows at a time; XCDs as above (1024 x 50 001 bf16: 44
// and 27 us).
template <class T, int G, bool SHIFT>
__global__ void __launch_bounds__(256) k_quant_unpack(QuantNet q, T* W) {
  const int lane = threadIdx.x & 63, b = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int nx = cdiv_dev(q.C, 64), item = xcd_item(blockIdx.x, nx * q.KB);
  if (item < 0) return;
  const int kb = item / nx, c = (item - kb * nx) * 64 + lane, k0 = kb * kQB + 32 * b;
  if (c >= q.C) return;
  constexpr int W16 = kQB / G * (SHIFT ? 2 : 1);
  const size_t block = (size_t)(c >> 4) * q.KB + kb;
  const u16* at = q.scale + (block * 16 + (c & 15)) * W16 + b / (G / 32) * (SHIFT ? 2 : 1);
  const float s = bf2f(at[0]), m = SHIFT ? bf2f(at[1]) : 0.f;
  uint32_t d[4];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    d[j] = reinterpret_cast<const uint32_t*>(q.code + block * 64 + j * 16 + (c & 15))[b];
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const int p = i & 1 ? 4 + i % 8 / 2 : i % 8 / 2;
    if (k0 + i < q.H)
      store_one(W + (size_t)(k0 + i) * q.C + c, fmaf((float)(d[i / 8] >> (4 * p) & 15u) - 8.f, s, m));
  }
}

// Eight codes less 8 as halves, exact: 0x6400 | q is 1024 + q, 0x6400 | q << 4 is
// 1024 + 16 q.  Nine instructions, where the bound by memory leaves about 26 for
// eight weights.  Codes left as 0 .. 15, in the bits of subnormal halves, take five,
// and 8 times the sum of x off afterwards: 16 x 128 000 x 2048 in 35.1 us instead of
// 36.1, but the sums are four times as large, and y's error was 3.5e-7 of it (fp32 x
// 9e-7) instead of 6e-8.  mask and magic are registers, so that one instruction takes
// both.
struct QuantBits {
  uint32_t low = 0x000f000fu, high = 0x00f000f0u, magic = 0x64006400u;
  __device__ __forceinline__ QuantBits() { asm("" : "+s"(low), "+s"(high), "+v"(magic)); }
};
__device__ __forceinline__ h8 halves(uint32_t w, const QuantBits& k) {
  const h2 a = {(_Float16)-1032.f, (_Float16)-1032.f}, f = {(_Float16)0.0625f, (_Float16)0.0625f},
           g = {(_Float16)-72.f, (_Float16)-72.f};
  auto at = [&](uint32_t v, uint32_t mask) { return __builtin_bit_cast(h2, (v & mask) | k.magic); };
  const uint32_t v = w >> 8;
  const h2 v0 = at(w, k.low) + a, v1 = __builtin_elementwise_fma(at(w, k.high), f, g);
  const h2 v2 = at(v, k.low) + a, v3 = __builtin_elementwise_fma(at(v, k.high), f, g);
  return h8{v0.x, v0.y, v1.x, v1.y, v2.x, v2.y, v3.x, v3.y};
}

// The rows' side of the product.  With X the sum of a group's x,
//   sum x What = sum over groups of s (sum x (q - 8)) + m X.
// x is scaled by a power of two 2^up for each row and block of 128 columns, so that
// the block's largest finite value lies in 2^14 .. 2^15: a half then holds what a bf16
// has, but that values below 2^-31 of the block's largest are off by up to half a
// half's smallest step, 2^-25, which is 2^-39 of the largest (less than an fp32 sum
// keeps of them).  An fp32 x is the sum of two halves: what the first leaves is at most
// 2^12 steps of x's last bit and the second holds 11 bits of it, so that one step,
// 2^-23 of x, may be lost, or the same 2^-39 of the largest where that is more (below
// some 2^-16 of it).  Products of halves and codes are exact, their sums are fp32.
//   LDS: xh [KC][parts][4 b][4 j][rows] of 16 bytes, xs [KC][16] = 2^-up,
//   with shifts xg [KC][groups][16] = X.

template <class X>
__device__ __forceinline__ void quant_load8(const X* __restrict__ x, int H, int k, float (&v)[8]) {
  if (k + 8 <= H) {   // at any address that is aligned to its elements
    if constexpr (sizeof(X) == 4) {
      typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
      const f4 a = *reinterpret_cast<const f4*>(x + k), b = *reinterpret_cast<const f4*>(x + k + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = a[i], v[4 + i] = b[i];
    } else {
      typedef u16 s8 __attribute__((ext_vector_type(8), aligned(2)));
      const s8 a = *reinterpret_cast<const s8*>(x + k);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = bf2f(a[i]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = k + i < H ? load_one(x + k + i) : 0.f;
  }
}

template <class X, int G, bool SHIFT, int R>
__device__ __forceinline__ void quant_put(const float (&v)[8], int o, int r, int kb, int rows, uint4* xh, float* xs,
                                          float* xg) {
  constexpr int P = sizeof(X) == 4 ? 2 : 1, NS = kQB / G;
  uint32_t top = 0;
  float sum = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t a = __float_as_uint(v[i]) & 0x7fffffffu;
    top = max(top, a < 0x7f800000u ? a : 0u);
    if (SHIFT) sum += v[i];
  }
#pragma unroll
  for (int d = 1; d < 16; d <<= 1) {
    top = max(top, (uint32_t)__shfl_xor((int)top, d, 16));
    if (SHIFT && d * 8 < G) sum += __shfl_xor(sum, d, 16);
  }
  // 2^126 at most: values below 2^-112 are whole steps of 2^-149, which are halves then
  const int e = max((int)(top >> 23) - 127, -112), up = top ? 14 - e : 0;
  uint32_t hi[4], lo[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    h2 h, l;
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const float t = ldexpf(v[2 * i + z], up);
      h[z] = (_Float16)t;
      l[z] = fabsf(t) < INFINITY ? (_Float16)(t - (float)h[z]) : (_Float16)0.f;
    }
    hi[i] = __builtin_bit_cast(uint32_t, h);
    lo[i] = __builtin_bit_cast(uint32_t, l);
  }
  // columns 8 o ..: dword b = o / 4 of lane group j = o % 4
  uint4* at = xh + ((size_t)kb * P * 16 + o) * rows + r;
  at[0] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
  if (P == 2) at[16 * rows] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
  if (o == 0) xs[kb * R + r] = ldexpf(1.f, -up);
  if (SHIFT && o % (G / 8) == 0) xg[(kb * NS + o / (G / 8)) * R + r] = sum;
}

// Blocks kb0 .. kb0 + nkb of all rows; a row's block to sixteen lanes, eight columns
// each, two such blocks in flight.
template <class X, int G, bool SHIFT, int R>
__device__ __forceinline__ void quant_stage(const X* __restrict__ x, int H, int rows, int kb0, int nkb, uint4* xh,
                                            float* xs, float* xg) {
  const int units = rows * nkb * 16, step = blockDim.x;
  for (int u = threadIdx.x; u < units; u += 2 * step) {
    float v[2][8];
    int r[2], kb[2];
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const int rb = min(u + z * step, units - 1) >> 4;
      kb[z] = rb / rows;
      r[z] = rb - kb[z] * rows;
      quant_load8(x + (size_t)r[z] * H, H, (kb0 + kb[z]) * kQB + 8 * (u & 15), v[z]);
    }
#pragma unroll
    for (int z = 0; z < 2; ++z)
      if (u + z * step < units) quant_put<X, G, SHIFT, R>(v[z], u & 15, r[z], kb[z], rows, xh, xs, xg);
  }
}

// y[rows, C] = x What + bias.  A workgroup of sixteen wavefronts has up to 16 RT rows
// of x (KC blocks of them at a time) in LDS and goes through groups of tiles; S
// wavefronts share a tile, each S-th block to one, and join their sums in LDS.  Each
// wavefront keeps PF blocks of codes in flight, over the ends of tiles.  The words
// are the rows of the matrix instruction's result, so that a lane has four adjacent
// ones of a row of y, one store: with four stores of a word each, the next blocks
// waited for them (16 x 128 000 x 2048: 43 us, 37 so).
// Bound by memory, the codes once: 16 x 128 000 x 2048 in 36 us (143 MB, 4.0 TB/s), of
// which reading the codes alone takes 28; 4 x 50 001 x 1024 in 10 (30 MB); below some
// 10 MB by latency (1 x 10 000 x 512 in 4.5).  fp32 rows have two halves a value: 42 us
// and 13.  Two forms are far from the codes' bytes: more than 16 rows, whose groups each
// make halves of the codes (64 x 32 000 x 2048 in 31 us, fp32 36, 42 MB), and rows that
// are not in LDS whole, which are staged anew for every group of tiles (16 x 32 000 x
// 4096 fp32 in 31 us, 70 MB; bf16, which fits, 25).
struct QuantJob {
  QuantNet q;
  const void* x;
  const float* bias;
  void* y;
  int n, KC, S, groups, ybf;
};

template <class X, int G, bool SHIFT, int RT>
__global__ void __launch_bounds__(64 * kQW) k_quant_product(QuantJob a) {
  constexpr int P = sizeof(X) == 4 ? 2 : 1, NS = kQB / G, W16 = NS * (SHIFT ? 2 : 1), PF = 2, R = kQR * RT;
  extern __shared__ uint4 lds[];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r0 = blockIdx.y * R, rows = min(R, a.n - r0);
  uint4* xh = lds;
  float* xs = reinterpret_cast<float*>(lds + (size_t)a.KC * P * 16 * rows);
  float* xg = xs + a.KC * R;
  v4f* red = reinterpret_cast<v4f*>(xg + (SHIFT ? a.KC * NS * R : 0));   // [kQW][RT][64]
  const X* x = (const X*)a.x + (size_t)r0 * a.q.H;
  const int KB = a.q.KB, T = a.q.T, S = a.S, ks = w % S, tw = w / S, per = kQW / S;
  const int steps = (KB + S - 1) / S, cstep = a.KC / S;   // blocks of a wavefront: of a tile, of a chunk
  const int mine = (a.groups - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;   // groups of tiles
  const int items = mine * steps, j = lane >> 4;
  int row[RT];
#pragma unroll
  for (int k = 0; k < RT; ++k) row[k] = min(k * kQR + (lane & 15), rows - 1);
  struct Block {
    uint4 c;
    uint32_t s[2 * W16];   // of this lane's four words
  } ring[PF];
  int ls = 0, lg = 0;   // the next block to ask for; past the last one, it again
  auto load = [&](Block& f) {
    const int kb = min(ls * S + ks, KB - 1), t = min(((int)blockIdx.x + lg * (int)gridDim.x) * per + tw, T - 1);
    const size_t block = (size_t)t * KB + kb;
    f.c = a.q.code[block * 64 + lane];
    __builtin_memcpy(f.s, __builtin_assume_aligned(a.q.scale + (block * 16 + 4 * j) * W16, 8), 8 * W16);
    if (++ls == steps) {
      ls = 0;
      lg = min(lg + 1, mine - 1);
    }
  };
#pragma unroll
  for (int u = 0; u < PF; ++u) load(ring[u]);
  const uint4* frag[RT];   // this lane's place in a dword's fragment of each sixteen rows
#pragma unroll
  for (int k = 0; k < RT; ++k) frag[k] = xh + j * rows + row[k];
  const QuantBits bits;
  v4f acc[RT] = {};
  int step = 0, cs = 0, grp = 0;
  for (int it0 = 0; it0 < items; it0 += PF) {
#pragma unroll
    for (int u = 0; u < PF; ++u) {
      if (it0 + u >= items) break;
      if (cs == 0 && (it0 + u == 0 || a.KC < KB)) {
        if (it0 + u > 0) __syncthreads();   // the last chunk has been read
        const int kb0 = step * S;
        quant_stage<X, G, SHIFT, R>(x, a.q.H, rows, kb0, min(a.KC, KB - kb0), xh, xs, xg);
        __syncthreads();
      }
      if (step * S + ks < KB) {
        const int kc = cs * S + ks;
        const uint32_t d[4] = {ring[u].c.x, ring[u].c.y, ring[u].c.z, ring[u].c.w};
        float f[RT];
#pragma unroll
        for (int k = 0; k < RT; ++k) f[k] = xs[kc * R + row[k]];
#pragma unroll
        for (int g = 0; g < NS; ++g) {
          v4f part[RT][P] = {};   // small halves apart: the instruction drops bits of theirs below a large sum
#pragma unroll
          for (int b = g * (4 / NS); b < (g + 1) * (4 / NS); ++b) {
            const h8 c8 = halves(d[b], bits);
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
              for (int k = 0; k < RT; ++k)
                part[k][p] = __builtin_amdgcn_mfma_f32_16x16x32_f16(
                    c8, __builtin_bit_cast(h8, frag[k][((kc * P + p) * 4 + b) * 4 * rows]), part[k][p], 0, 0, 0);
          }
#pragma unroll
          for (int k = 0; k < RT; ++k) {
            if (P == 2) part[k][0] += part[k][P - 1];
            const float X1 = SHIFT ? xg[(kc * NS + g) * R + row[k]] : 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {   // word i's numbers: halves W16 i and on
              const int at = W16 * i + g * (SHIFT ? 2 : 1);
              const uint32_t s = ring[u].s[at / 2];
              acc[k][i] = fmaf(__uint_as_float(at & 1 ? s & 0xffff0000u : s << 16), f[k] * part[k][0][i], acc[k][i]);
              if (SHIFT) acc[k][i] = fmaf(__uint_as_float(s & 0xffff0000u), X1, acc[k][i]);
            }
          }
        }
      }
      load(ring[u]);
      if (++cs == cstep) cs = 0;
      if (++step < steps) continue;
      // the tile is done
      step = cs = 0;
      const int t = ((int)blockIdx.x + grp++ * (int)gridDim.x) * per + tw;
      if (S > 1) {
        __syncthreads();
        if (ks > 0)
#pragma unroll
          for (int k = 0; k < RT; ++k) red[(w * RT + k) * 64 + lane] = acc[k];
        __syncthreads();
        if (ks == 0)
          for (int o = 1; o < S; ++o)
#pragma unroll
            for (int k = 0; k < RT; ++k) acc[k] += red[((w + o) * RT + k) * 64 + lane];
      }
      const int c = t * 16 + 4 * j;
      if (ks == 0 && t < T && c < a.q.C) {
        const bool whole = c + 4 <= a.q.C;
        float bias[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) bias[i] = a.bias && (whole || c + i < a.q.C) ? a.bias[c + i] : 0.f;
#pragma unroll
        for (int k = 0; k < RT; ++k) {
          if (k * kQR + (lane & 15) >= rows) continue;
          const size_t at = (size_t)(r0 + row[k]) * a.q.C + c;
          float v[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] = acc[k][i] + bias[i];
          if (whole) {   // at any address that is aligned to its elements
            typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
            typedef uint32_t u2 __attribute__((ext_vector_type(2), aligned(2)));
            if (a.ybf) *reinterpret_cast<u2*>((u16*)a.y + at) = u2{f2bf2(v[0], v[1]), f2bf2(v[2], v[3])};
            else *reinterpret_cast<f4*>((float*)a.y + at) = f4{v[0], v[1], v[2], v[3]};
          } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (c + i < a.q.C) a.ybf ? store_one((u16*)a.y + at + i, v[i]) : store_one((float*)a.y + at + i, v[i]);
          }
        }
      }
#pragma unroll
      for (int k = 0; k < RT; ++k) acc[k] = v4f{0.f, 0.f, 0.f, 0.f};
    }
  }
}

cavs_status quant_args(cavs_ctx* ctx, const cavs_quant* q) {
  if (!q) return fail(ctx, CAVS_ERR_ARG, "null weights");
  if (q->H <= 0 || q->C <= 0) return fail(ctx, CAVS_ERR_ARG, "bad H/C");
  if (q->group != 32 && q->group != 64 && q->group != 128)
    return fail(ctx, CAVS_ERR_ARG, "group=%d: 32, 64 or 128", q->group);
  if (q->shift != 0 && q->shift != 1) return fail(ctx, CAVS_ERR_ARG, "shift=%d: 0 or 1", q->shift);
  if (q->H > kQuantMaxH || q->C > kQuantMaxC)
    return fail(ctx, CAVS_ERR_UNSUPPORTED, "H=%d, C=%d: at most %d, %d", q->H, q->C, kQuantMaxH, kQuantMaxC);
  return CAVS_OK;
}

size_t code_bytes(const cavs_quant* q) {
  return (size_t)cdiv(q->C, 16) * cdiv(q->H, kQB) * 1024;
}

QuantNet quant_net(const cavs_quant* q, const void* data) {
  QuantNet n{q->H, q->C, cdiv(q->C, 16), cdiv(q->H, kQB), (const uint4*)data,
             (const u16*)((const char*)data + code_bytes(q))};
  return n;
}

cavs_status quant_data(cavs_ctx* ctx, const void* data) {
  if (!data) return fail(ctx, CAVS_ERR_ARG, "data is required");
  if (((uintptr_t)data & 15) != 0) return fail(ctx, CAVS_ERR_ARG, "data must be aligned to 16 bytes");
  return CAVS_OK;
}

cavs_status quant_type(cavs_ctx* ctx, int type, const void* p, const char* name) {
  if (type != CAVS_T_F32 && type != CAVS_T_BF16) return fail(ctx, CAVS_ERR_ARG, "unknown element type");
  if (!p) return fail(ctx, CAVS_ERR_ARG, "%s is required", name);
  if (((uintptr_t)p & (type == CAVS_T_BF16 ? 1 : 3)) != 0)
    return fail(ctx, CAVS_ERR_ARG, "%s is not aligned to its elements", name);
  return CAVS_OK;
}

template <class F>
void by_group(const cavs_quant* q, F f) {
  auto g = [&](auto shift) {
    if (q->group == 32) f(std::integral_constant<int, 32>{}, shift);
    else if (q->group == 64) f(std::integral_constant<int, 64>{}, shift);
    else f(std::integral_constant<int, 128>{}, shift);
  };
  q->shift ? g(std::true_type{}) : g(std::false_type{});
}

template <class F>
void by_element(int type, F f) {
  type == CAVS_T_BF16 ? f(u16{}) : f(float{});
}

// At most kQuantStep rows of x, whose groups of sixteen are a grid's second dimension.
constexpr int kQuantStep = 1 << 19;
void quant_product_launch(cavs_ctx* ctx, const cavs_quant* q, int x_type, const void* x, int n, const float* bias,
                          int y_type, void* y) {
  QuantJob a{quant_net(q, q->data), x, bias, y, n};
  a.ybf = y_type == CAVS_T_BF16;
  const int P = x_type == CAVS_T_F32 ? 2 : 1, T = a.q.T, KB = a.q.KB;
  size_t shmem;
  dim3 grid;
  // wavefronts of a tile: as many as leave each of 2048 something to do; two of long
  // tiles, whose blocks are then read in the order of memory by neighbours (16 x
  // 128 000 x 2048: 37.0 us with one, 35.8 with two, 36.1 with four; of 1024: one)
  auto plan = [&](int rt) {
    const int rows = cdiv(n, kQR * rt);
    const size_t block = (size_t)P * 256 * std::min(n, kQR * rt) + 4 * kQR * rt * (1 + (q->shift ? kQB / q->group : 0));
    a.S = KB >= 16 ? 2 : 1;
    const size_t sums = (size_t)kQW * rt * 1024;
    while (a.S < 8 && a.S < KB && (long)T * a.S * rows < 2048 && 2 * a.S * block + sums <= kQLds) a.S *= 2;
    const size_t red = a.S > 1 ? sums : 0;
    a.KC = std::min(cdiv(KB, a.S), (int)((kQLds - red) / block) / a.S) * a.S;
    a.groups = cdiv(T, kQW / a.S);
    shmem = a.KC * block + red;
    // a workgroup per CU; the groups of rows of a tile on one XCD
    grid = dim3(std::min(a.groups, (int)align_up(cdiv(256, rows), 8)), rows);
  };
  // 32 rows of x to a workgroup where there are tiles for all wavefronts without
  // sharing them and the rows are short enough to be in LDS once for all tiles: the
  // codes become halves once for them (64 x 50 001 x 1024 in bf16 27 us with 16 rows and
  // 21 with 32, 64 x 30 000 16.8 and 14.9; but 64 x 10 000 x 512 in fp32 8.6 and 9.5,
  // 64 x 32 000 x 2048 32 and 38)
  plan(2);
  const bool two = n > kQR && KB < 16 && a.S == 1 && a.KC == KB;
  if (!two) plan(1);
  by_group(q, [&](auto g, auto shift) {
    by_element(x_type, [&](auto t) {
      using X = decltype(t);
      auto launch = [&](auto kernel) {
        if (shmem > 64 << 10)
          (void)hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)shmem);
        CAVS_LAUNCH("k_quant_product", kernel, grid, dim3(64 * kQW), shmem, ctx->stream, a);
      };
      two ? launch(k_quant_product<X, g(), shift(), 2>) : launch(k_quant_product<X, g(), shift(), 1>);
    });
  });
}

}  // namespace

size_t quant_bytes(const cavs_quant* q) {
  if (quant_args(nullptr, q) != CAVS_OK) return 0;
  const size_t blocks = (size_t)cdiv(q->C, 16) * cdiv(q->H, kQB);
  return code_bytes(q) + blocks * 16 * (kQB / q->group) * (q->shift ? 4 : 2);
}

cavs_status quant_pack_run(cavs_ctx* ctx, const cavs_quant* q, int w_type, const void* W, void* data) {
  cavs_status st = quant_args(ctx, q);
  if (st == CAVS_OK) st = quant_type(ctx, w_type, W, "W");
  if (st == CAVS_OK) st = quant_data(ctx, data);
  if (st != CAVS_OK) return st;
  const QuantNet n = quant_net(q, data);
  by_group(q, [&](auto g, auto shift) {
    by_element(w_type, [&](auto t) {
      using T = decltype(t);
      CAVS_LAUNCH("k_quant_pack", (k_quant_pack<T, g(), shift()>), dim3(xcd_grid(cdiv(n.C, 64) * n.KB)), dim3(512), 0,
                  ctx->stream, n, (const T*)W, (uint4*)data, (u16*)((char*)data + code_bytes(q)));
    });
  });
  CAVS_LAUNCH_CHECK(ctx);
  return CAVS_OK;
}

cavs_status quant_unpack_run(cavs_ctx* ctx, const cavs_quant* q, int w_type, void* W) {
  cavs_status st = quant_args(ctx, q);
  if (st == CAVS_OK) st = quant_type(ctx, w_type, W, "W");
  if (st == CAVS_OK) st = quant_data(ctx, q->data);
  if (st != CAVS_OK) return st;
  const QuantNet n = quant_net(q, q->data);
  by_group(q, [&](auto g, auto shift) {
    by_element(w_type, [&](auto t) {
      using T = decltype(t);
      CAVS_LAUNCH("k_quant_unpack", (k_quant_unpack<T, g(), shift()>), dim3(xcd_grid(cdiv(n.C, 64) * n.KB)), dim3(256), 0,
                  ctx->stream, n, (T*)W);
    });
  });
  CAVS_LAUNCH_CHECK(ctx);
  return CAVS_OK;
}

cavs_status quant_product_run(cavs_ctx* ctx, const cavs_quant* q, int x_type, const void* x, int n,
                              const float* bias, int y_type, void* y) {
  cavs_status st = quant_args(ctx, q);
  if (st != CAVS_OK) return st;
  if (n < 0) return fail(ctx, CAVS_ERR_ARG, "bad n");
  if (n > kQuantMaxN) return fail(ctx, CAVS_ERR_UNSUPPORTED, "n=%d: at most %d", n, kQuantMaxN);
  if ((x_type != CAVS_T_F32 && x_type != CAVS_T_BF16) || (y_type != CAVS_T_F32 && y_type != CAVS_T_BF16))
    return fail(ctx, CAVS_ERR_ARG, "unknown element type");
  if (n == 0) return CAVS_OK;
  st = quant_type(ctx, x_type, x, "x");
  if (st == CAVS_OK) st = quant_type(ctx, y_type, y, "y");
  if (st == CAVS_OK) st = quant_data(ctx, q->data);
  if (st != CAVS_OK) return st;
  if (((uintptr_t)bias & 3) != 0) return fail(ctx, CAVS_ERR_ARG, "bias is not aligned to its elements");
  const size_t xs = (size_t)q->H * (x_type == CAVS_T_BF16 ? 2 : 4), ys = (size_t)q->C * (y_type == CAVS_T_BF16 ? 2 : 4);
  for (int at = 0; at < n; at += kQuantStep)
    quant_product_launch(ctx, q, x_type, (const char*)x + at * xs, std::min(n - at, kQuantStep), bias, y_type,
                         (char*)y + at * ys);
  CAVS_LAUNCH_CHECK(ctx);
  return CAVS_OK;
}

}  // namespace cavs
