// What the kernels of the softmax attention over another set of tokens (attn.hip, attn_grad.hip) share.
//
// Rows. The G = H / Hkv query heads that share a key head are the rows of one problem: row r = i G + g is query
// i of head hk G + g, R = Nq G rows per (b, key head). A tile of rows then reads its keys once for all of
// them (a single token's G heads are one tile), and its queries' positions stay close together, which is
// what a causal tile's key range goes by.
// Keys. Row i sees the keys below limit(i): n = kv_len[b] (clamped to [0, Nk]), and with the causal mask at
// most i + n - Nq + 1 (the last query sees all n keys). A row with limit <= 0 sees none: its output is zero, its
// log-sum-exp -inf, and it has no part in any gradient.
#pragma once

#include "common.h"
#include "launch.h"

namespace rola {

struct View {
  char* p;
  long b, h, n;  // byte strides
};

struct AttnCall {
  int Hkv, G, Nq, Nk, causal;
  const int32_t* kv_len;
  float scale, scale_log2;
  View Q, K, V, O;
};

__device__ __forceinline__ int attn_keys(const AttnCall& a, int b) {
  return a.kv_len ? max(0, min(a.kv_len[b], a.Nk)) : a.Nk;
}
// Keys that query i sees (may be negative).
__device__ __forceinline__ int attn_limit(const AttnCall& a, int n, int i) {
  return a.causal ? min(n, i + n - a.Nq + 1) : n;
}

inline View view_of(const HeadView& v, bool bf) {
  const long e = bf ? 2 : 4;
  return View{(char*)const_cast<void*>(v.p), v.b * e, v.h * e, v.n * e};
}
inline AttnCall attn_call(const AttnShape& s, const HeadView& Q, const HeadView& K, const HeadView& V,
                          const HeadView& O, const int32_t* kv_len, float scale) {
  return AttnCall{s.Hkv, s.H / s.Hkv, s.Nq, s.Nk, s.causal, kv_len, scale, scale * 1.4426950408889634f,
                  view_of(Q, s.bf16), view_of(K, s.bf16), view_of(V, s.bf16), view_of(O, s.bf16)};
}

__device__ __forceinline__ f32x16 mfma_bf16(const bf16x8& a, const bf16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mfma_f32(float a, float b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// How a pass over (b, key head, tile) is cut into workgroups. The first `whole` tiles, whole rounds of the
// workgroups that the chip holds, have one each; the `left` ones of the last, partial round are given to `splits`
// workgroups each, which take a part of the tile's walk and leave partial sums, so that the chip is full to the
// end (8400 tokens, 12 heads: 792 tiles of dK/dV on 256 CUs are three rounds and 24 tiles). A causal pass has
// walks of all lengths and no rounds, so it is cut only where the tiles are fewer than one round.
struct Cut {
  int tiles, bh, whole, splits, total, causal;
};
struct Part {
  int tile, b, hk;
  int split, splits;
  int left;  // which of the cut tiles, -1 for a whole one
  long bh;
};
// The tile at a place in the order: heads one after the other, so that an XCD's share is whole heads; in a
// causal call a head's long and short walks by turns, so that every share has as much work. Samples of different
// lengths are not dealt out: a share lies within one or two of them. (Two samples of 512 and 73 keys with 12 heads and
// 32760 queries each: 12288 steps on four XCDs and 2304 on the other four, the mean being 7296. Eight caches of 32760
// to 4679 keys: one on each XCD, the first with 1.75 times the mean.)
__device__ __forceinline__ void cut_tile(const Cut& c, int idx, int* tile, long* bh) {
  const int t = idx % c.tiles;
  *bh = idx / c.tiles;
  *tile = !c.causal ? t : t % 2 ? t / 2 : c.tiles - 1 - t / 2;
}
// And the place of a tile.
__device__ __forceinline__ int cut_place(const Cut& c, int tile, long bh) {
  int t = tile;
  if (c.causal) t = 2 * (c.tiles - 1 - tile) < c.tiles ? 2 * (c.tiles - 1 - tile) : 2 * tile + 1;
  return (int)(bh * c.tiles + t);
}
__device__ __forceinline__ Part part_of(const Cut& c, int Hkv, int wg) {
  Part p;
  int idx;
  if (wg < c.whole) {
    idx = xcd_remap(wg, c.whole);
    p.split = 0, p.splits = 1, p.left = -1;
  } else {
    const int m = xcd_remap(wg - c.whole, c.total - c.whole);
    p.left = m / c.splits;
    p.split = m % c.splits, p.splits = c.splits;
    idx = c.whole + p.left;
  }
  cut_tile(c, idx, &p.tile, &p.bh);
  p.b = (int)(p.bh / Hkv);
  p.hk = (int)(p.bh % Hkv);
  return p;
}
// slots: workgroups that the chip holds; steps: of a whole walk; step_us: what one lasts; part_bytes: partial sums
// of one part; least: steps that a part has at least.
inline Cut make_cut(int tiles, int bh, bool causal, int slots, int steps, double step_us, double part_bytes,
                    int least) {
  Cut c{tiles, bh, 0, 1, 0, causal};
  const long all = (long)tiles * bh;
  long left = all % slots;
  if (causal && all >= slots) left = 0;
  if (left > 0) {
    // rounds of a part's walk and its set-up (about two steps), then the sums written, read and one more launch
    double best = -1;
    for (int s = 1; s <= 64 && (s == 1 || (steps + s - 1) / s >= least); ++s) {
      const double rounds = (double)((left * s + slots - 1) / slots);
      double us = rounds * ((steps + s - 1) / s + 2) * step_us;
      if (s > 1) us += 5 + 2 * left * s * part_bytes / 4e6;
      if (best < 0 || us < 0.97 * best) best = us, c.splits = s;
    }
  }
  if (c.splits == 1) left = 0;
  c.whole = (int)(all - left);
  c.total = (int)(c.whole + left * c.splits);
  return c;
}
// fp32: 16-row tiles whose walk four waves share, where tiles of 64 rows are so few that latency bounds them: below one
// tile per CU (2048 x 2048, 12 heads, 384 tiles, d 128: forward 501 us with 16 rows, 341 with 64), and below an amount of
// work B H Nq Nk d, as every 16 rows read the walk again from memory. Calls in us with 16 rows and with 64:
//   forward, d 128: 12 x 500 x 1100 (0.8e9) 80 and 86; 2700 x 2700 (0.9e9) 91 and 80; 2 x 4000 x 4000 (4e9) 298 and
//   220. At d 64 a tile's walk is half as long in bytes and 16 rows are the faster up to the 2e9 that was tried
//   (2 x 4000 x 4000: 115 and 127).
//   gradients: 4 x 3000 x 300, d 128 (0.5e9) 126 and 145; 3 x 2000 x 1000, d 128 (0.8e9) 206 and 182; 2 x 4000 x 4000,
//   d 64 (2e9) 373 and 330. Not in order at d 64: 6 x 1500 x 1000 (0.6e9) 148 and 139, 8 x 600 x 6000 (1.8e9) 305 and 320.
// All pairs count, also those that a causal mask or a sample's length leaves out.
constexpr double kFewForward = 0.9e9, kFewGrad = 0.55e9;
inline double attn_work(const AttnShape& s) { return (double)s.B * s.H * s.Nq * s.Nk * s.d; }
inline bool f32_few(long tiles, long bh) { return tiles * bh < kCus; }
inline long cut_left(const Cut& c) { return c.splits > 1 ? (c.total - c.whole) / c.splits : 0; }

// Query head rows of one (b, key head): row r is query r / G of head hk G + r % G.
struct RowBase {
  char* p;  // query 0 of the first head
  long h, n;
  int G;
};
__device__ __forceinline__ RowBase row_base(const View& v, int b, int hk, int G) {
  return RowBase{v.p + b * v.b + (long)hk * G * v.h, v.h, v.n, G};
}
__device__ __forceinline__ char* row_at(const RowBase& v, int r) {
  if (v.G == 1) return v.p + (long)r * v.n;  // (uniform; a division costs twenty instructions)
  const int i = r / v.G;
  return v.p + (long)i * v.n + (long)(r - i * v.G) * v.h;
}

// Stores the wave's 32 rows from the accumulator layout of a 32x32 tile set (lane: row l%32, channels
// 32 w + 8 j + 4 hh ..), scaled by f and rounded to bf16, through 8 KB of LDS of its own: whole rows of 256
// bytes, four to a store, instead of 16-byte pieces of 32 rows (text cross-attention of 2 x 32760 queries, 512 and
// 73 keys: forward 235 -> 219 us).
__device__ __forceinline__ void rows_from_acc(char* tile, const f32x16 (&acc)[4], float f, const RowBase& v,
                                              int row0, int rows, int lane) {
  const int hh = lane / 32, own = lane % 32;
#pragma unroll
  for (int w = 0; w < 4; ++w)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      bf16x4 o;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = (bf16)(acc[w][4 * j + e] * f);
      *reinterpret_cast<bf16x4*>(tile + own * 256 + (((4 * w + j) ^ bw_swizzle(own)) << 4) + 8 * hh) = o;
    }
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int x = 0; x < 8; ++x) {
    const int row = 4 * x + lane / 16, c = lane % 16;
    const uint4 o = *reinterpret_cast<const uint4*>(tile + row * 256 + ((c ^ bw_swizzle(row)) << 4));
    if (row0 + row < rows) *reinterpret_cast<uint4*>(row_at(v, row0 + row) + 16 * c) = o;
  }
}

// s_waitcnt vmcnt(N), the other counters free.
template <int N>
__device__ __forceinline__ void wait_vm() {
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}

// Sum of x over the lanes l and l ^ 32.
__device__ __forceinline__ float halves_sum(float x) {
  const auto v = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(v[0]) + __uint_as_float(v[1]);
}
__device__ __forceinline__ float halves_max(float x) {
  const auto v = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(v[0]), __uint_as_float(v[1]));
}

// Reference max of a row that has seen no key yet: below every finite score, and finite, so that a hidden
// key's exp2(-inf - m) is zero and not NaN.
constexpr float kNoMax = -3e38f;
// 1 / l and log2 of a row's denominator, from its maximum m and sum l; of a row that has seen no key (l is the zero it
// started from) 0 and -inf, the mark by which the gradients leave it out. A NaN or +inf score makes l NaN, and
// both results. (By its bits: the library is built with NaN compares free to go either way.)
__device__ __forceinline__ float row_inverse(float l) { return __float_as_uint(l) == 0 ? 0.f : 1.f / l; }
__device__ __forceinline__ float row_lse(float m, float l) {
  return __float_as_uint(l) == 0 ? -__builtin_inff() : m + __log2f(l);
}
__device__ __forceinline__ bool saw_no_key(float lse) { return __float_as_uint(lse) == 0xff800000u; }  // -inf

// ---- fp32 tiles -------------------------------------------------------------------------------------
// On v_mfma_f32_16x16x4_f32 (A: row l%16, k = l/16; B: column l%16, k = l/16; D: column l%16, rows
// 4(l/16) + i) with 16-row tiles:
//   f32_rows   X Y^T, X the tile, Y a row per lane in registers; step s of lane group g contracts channel
//              g D/4 + s, so that both sides are read as 16-byte pieces;
//   f32_cols   acc += X^T p, p[i] the value of tile row 4g + i (where f32_rows leaves it); row l%16 of channel
//              tile 4s + e is channel 64s + 4 (l%16) + e, again whole pieces, side by side over the lanes.
template <int D>
__device__ __forceinline__ f32x4 f32_rows(const float4 (&x)[D / 16], const float4 (&y)[D / 16]) {
  f32x4 s0 = f32x4{0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
  for (int s = 0; s < D / 16; ++s) {
    s0 = mfma_f32(x[s].x, y[s].x, s0);
    s1 = mfma_f32(x[s].y, y[s].y, s1);
    s0 = mfma_f32(x[s].z, y[s].z, s0);
    s1 = mfma_f32(x[s].w, y[s].w, s1);
  }
  return s0 + s1;
}
template <int D>
__device__ __forceinline__ void f32_cols(const float4 (&x)[4][D / 64], const float (&p)[4], f32x4 (&acc)[D / 16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int s = 0; s < D / 64; ++s) {
      acc[4 * s] = mfma_f32(x[i][s].x, p[i], acc[4 * s]);
      acc[4 * s + 1] = mfma_f32(x[i][s].y, p[i], acc[4 * s + 1]);
      acc[4 * s + 2] = mfma_f32(x[i][s].z, p[i], acc[4 * s + 2]);
      acc[4 * s + 3] = mfma_f32(x[i][s].w, p[i], acc[4 * s + 3]);
    }
}
// The operands from a tile in LDS, rows padded to D + 4 floats.
template <int D>
__device__ __forceinline__ f32x4 f32_rows(const float* tile, const float4 (&y)[D / 16], int lane) {
  const float* row = tile + (lane % 16) * (D + 4) + (lane / 16) * (D / 4);
  float4 x[D / 16];
#pragma unroll
  for (int s = 0; s < D / 16; ++s) x[s] = *reinterpret_cast<const float4*>(row + 4 * s);
  return f32_rows<D>(x, y);
}
template <int D>
__device__ __forceinline__ void f32_cols(const float* tile, const float (&p)[4], f32x4 (&acc)[D / 16],
                                         int lane) {
  const float* at = tile + 4 * (lane / 16) * (D + 4) + (lane % 16) * 4;
  float4 x[4][D / 64];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int s = 0; s < D / 64; ++s) x[i][s] = *reinterpret_cast<const float4*>(at + i * (D + 4) + 64 * s);
  f32_cols<D>(x, p, acc);
}
// The second operand from memory: a lane's pieces of rows row0 + 4 g + i, those past `last` re-read that one.
template <int D>
__device__ __forceinline__ void f32_pieces(const char* base, long stride, int row0, int last, int lane,
                                           float4 (&x)[4][D / 64]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const char* row = base + min(row0 + 4 * (lane / 16) + i, last) * stride;
#pragma unroll
    for (int s = 0; s < D / 64; ++s) x[i][s] = reinterpret_cast<const float4*>(row)[lane % 16 + 16 * s];
  }
}
// A lane's quarter of a row, for f32_rows.
template <int D>
__device__ __forceinline__ void f32_quarter(const char* row, int lane, float4 (&y)[D / 16]) {
  const float4* at = reinterpret_cast<const float4*>(row) + (lane / 16) * (D / 16);
#pragma unroll
  for (int s = 0; s < D / 16; ++s) y[s] = at[s];
}
// Adds up the accumulators of four waves for the same 16 rows, in order, through LDS [4][16][D + 4]: thread
// tid has channels (tid % 16) W .. of row tid / 16.
template <int D>
__device__ __forceinline__ void f32_join(float* lds, const f32x4 (&acc)[D / 16], int wave, int lane,
                                         float (&o)[D / 16]) {
  constexpr int W = D / 16;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int s = 0; s < W / 4; ++s)
      *reinterpret_cast<float4*>(lds + (wave * 16 + lane % 16) * (D + 4) + 64 * s + 4 * (4 * (lane / 16) + i)) =
          make_float4(acc[4 * s][i], acc[4 * s + 1][i], acc[4 * s + 2][i], acc[4 * s + 3][i]);
  __syncthreads();
#pragma unroll
  for (int k = 0; k < W; ++k) {
    o[k] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) o[k] += lds[(w * 16 + threadIdx.x / 16) * (D + 4) + (threadIdx.x % 16) * W + k];
  }
}
// Stores a row from f32_cols' accumulators (lane: row l%16, channels 64 s + 4 (4g + i) + e), scaled by f.
template <int D>
__device__ __forceinline__ void f32_store(char* row, const f32x4 (&acc)[D / 16], float f, int lane) {
  constexpr int W = D / 16;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int s = 0; s < W / 4; ++s)
      reinterpret_cast<float4*>(row)[16 * s + 4 * (lane / 16) + i] =
          make_float4(acc[4 * s][i] * f, acc[4 * s + 1][i] * f, acc[4 * s + 2][i] * f, acc[4 * s + 3][i] * f);
}

}  // namespace rola
