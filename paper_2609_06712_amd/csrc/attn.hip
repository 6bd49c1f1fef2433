// Softmax attention of Nq queries over Nk keys of another length, with key lengths per sample, the causal
// mask, key heads shared by groups of query heads, and tensors in place by strides (attn_common.h):
//   S = scale Q K^T over the visible keys, O = softmax(S) V, lse = log2 sum exp2(S log2e).
// One pass over the keys with a running maximum and sum per row. Bound by the matrix cores where rows are many
// (4 d operations per visible pair), by reading K and V once where they are few.
//
// bf16 (d 128), on v_mfma_f32_32x32x16_bf16, keys in sub-tiles of 32:
//   S^T = K Q^T     A = K rows from LDS, B = Q in registers; a lane has one row and 16 keys of it;
//   O^T = V^T P^T   A = V^T through the transposing LDS read, in the order the lane holds its keys.
// P is rounded to bf16 for that product (half a step, at most 2^-8 of a term, as the inputs); the row sum adds the
// probabilities before that rounding, so that lse is an fp32 value. O^T is rescaled only when a row's maximum
// grows by more than 2^8, which leaves the quotient as it is.
//   QW = 4: four waves of 32 rows each walk the keys together, three LDS stages, three workgroups per CU.
//   QW = 1: few rows (R <= 32): the four waves take every fourth sub-tile of the same rows through stages of
//           their own, without barriers, and add up through LDS.
// Measured in a kernel trace: 8400 x 8400, 12 heads 392 us (1.11 PFLOP/s, matrix cores busy 0.77 of the cycles); one
// token of 40 heads over 8 caches of 8 key heads, 32760 to 4679 keys, 135 us (613 MB: 4.5 TB/s) and 6 for the join.
// The tiles of rows that do not fill a round of the chip are cut over their keys (Cut); the partial results (fp32,
// with maximum and sum) are joined by attn_join_kernel in a fixed order.
//
// fp32 (d 64, 128), on fp32 matrix instructions (attn_common.h): workgroups of 64 rows, 16 per wave, or for few
// rows of 16 with the keys dealt over the waves.
#include <algorithm>

#include "attn_common.h"

namespace rola {
namespace {

constexpr float kTau = 8.f;      // log2 headroom before O is rescaled
constexpr int kKeys = 32;        // keys per sub-tile
constexpr int kTile = kKeys * 256;  // bytes of K or V of a sub-tile (bf16)

struct FwdArgs {
  AttnCall c;
  Cut cut;
  int R, rows;     // rows per key head, and per tile
  long heads;      // query heads, H
  float* lse;      // [B, H, Nq] or null
  float* part;     // of the cut tiles: O [left][splits][rows][d], and {max, sum} [left][splits][rows]
  float2* ml;
};

// V^T operand of a row-major [key][128] tile whose 16-byte chunks are swizzled by v_swizzle: as tr_frag, with
// one address per channel tile for both halves of a k-step (four registers less than bw_swizzle takes).
__device__ __forceinline__ int v_swizzle(int row) { return 2 * ((0x6530 >> (4 * (row & 3))) & 15); }
__device__ __forceinline__ int v_offset(int w, int lane) {
  const int i16 = lane % 16, row = 4 * (lane / 32) + i16 / 4, c = 2 * ((lane / 16) & 1) + ((i16 & 3) >> 1);
  return row * 256 + (((4 * w + c) ^ v_swizzle(row)) << 4) + 8 * (i16 & 1);
}
__device__ __forceinline__ bf16x8 v_frag(const char* tile, int off, int u) {
  const char* p = tile + off + 16 * u * 256;
  const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)p);
  const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(p + 8 * 256));
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

template <int QW>
__global__ __launch_bounds__(256, QW == 4 ? 3 : 1) void attn_bf16_kernel(const FwdArgs a) {
  constexpr int D = 128, STAGE = 2 * kTile;
  constexpr int NBUF = QW == 4 ? 3 : 2;
  constexpr int DPW = QW == 4 ? 2 : 8;         // 1 KB loads per wave, tensor and sub-tile
  constexpr int STEP = QW == 4 ? 1 : 4;        // sub-tiles between two of a wave's
  __shared__ __attribute__((aligned(1024))) char lds[(QW == 4 ? 1 : 4) * NBUF * STAGE];
  const AttnCall& c = a.c;
  const Part pt = part_of(a.cut, c.Hkv, blockIdx.x);
  const int wave = wave_uniform(threadIdx.x / 64), lane = threadIdx.x % 64, hh = lane / 32;
  const int n = attn_keys(c, pt.b);
  const int row0 = (pt.tile * QW + (QW == 4 ? wave : 0)) * 32;  // first row of this wave
  const int r = min(row0 + lane % 32, a.R - 1);
  const int lim = attn_limit(c, n, r / c.G);
  // least and greatest limit of the wave's rows, and the greatest of the workgroup's
  const int lim_lo = attn_limit(c, n, min(row0, a.R - 1) / c.G);
  const int lim_hi = row0 < a.R ? attn_limit(c, n, min(row0 + 31, a.R - 1) / c.G) : 0;
  const int end = max(0, attn_limit(c, n, min((pt.tile + 1) * 32 * QW - 1, a.R - 1) / c.G));
  const int all = (end + kKeys - 1) / kKeys, per = (all + pt.splits - 1) / pt.splits;
  const int t0 = pt.split * per, t1 = min(all, t0 + per);
  const int first = t0 + (QW == 4 ? 0 : wave);
  const int T = t1 > first ? (t1 - first + STEP - 1) / STEP : 0;  // this wave's sub-tiles

  const char* Kh = c.K.p + pt.b * c.K.b + pt.hk * c.K.h;
  const char* Vh = c.V.p + pt.b * c.V.b + pt.hk * c.V.h;
  // 1 KB load `x` of a wave fills tile rows 4 x .. 4 x + 3; lane l row l/16 at chunk l%16, swizzled.
  uint32_t dk[DPW], dv[DPW];
#pragma unroll
  for (int x = 0; x < DPW; ++x) {
    const int row = 4 * ((QW == 4 ? wave * DPW : 0) + x) + lane / 16;
    dk[x] = row * (uint32_t)c.K.n + (((lane % 16) ^ bw_swizzle(row)) << 4);
    dv[x] = row * (uint32_t)c.V.n + (((lane % 16) ^ v_swizzle(row)) << 4);
  }
  const uint32_t lds0 = lds_address(lds) + (QW == 4 ? 0 : wave * NBUF * STAGE);
  char* stages = lds + (QW == 4 ? 0 : wave * NBUF * STAGE);

  bf16x8 qf[8];
  {
    const char* q = row_at(row_base(c.Q, pt.b, pt.hk, c.G), r);
#pragma unroll
    for (int s = 0; s < 8; ++s) qf[s] = *reinterpret_cast<const bf16x8*>(q + 32 * s + 16 * hh);
    wait_vm<0>();
  }

  int vo[4];
  f32x16 acc[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) acc[w] = f32x16{}, vo[w] = v_offset(w, lane);
  float m = kNoMax, l = 0.f;

  auto issue = [&](int t, int buf) {  // sub-tile `t` of the wave's walk
    const int k0 = (first + t * STEP) * kKeys;
    const uint32_t dst = lds0 + buf * STAGE + (QW == 4 ? wave * DPW * 1024 : 0);
    const char* kb = Kh + (long)k0 * c.K.n;
    const char* vb = Vh + (long)k0 * c.V.n;
    if (k0 + kKeys <= n) {
#pragma unroll
      for (int x = 0; x < DPW; ++x) {
        dma16(kb, dk[x], dst + x * 1024);
        dma16(vb, dv[x], dst + kTile + x * 1024);
      }
    } else {  // rows past the last key re-read it; their probabilities are zero
#pragma unroll
      for (int x = 0; x < DPW; ++x) {
        const int row = 4 * ((QW == 4 ? wave * DPW : 0) + x) + lane / 16;
        const int back = max(row - (n - 1 - k0), 0);
        dma16(kb, dk[x] - back * (uint32_t)c.K.n, dst + x * 1024);
        dma16(vb, dv[x] - back * (uint32_t)c.V.n, dst + kTile + x * 1024);
      }
    }
  };

  int issued = 0;
#pragma unroll
  for (int j = 0; j < NBUF - 1; ++j)
    if (j < T) issue(j, j), ++issued;
  for (int t = 0; t < T;) {
#pragma unroll
    for (int j = 0; j < NBUF; ++j) {
      if (t >= T) break;
      if (NBUF > 2 && issued == t + NBUF - 1)
        wait_vm<2 * DPW * (NBUF - 2)>();
      else
        __builtin_amdgcn_s_waitcnt(0);
      if (QW == 4) __syncthreads();  // sub-tile t landed for every wave, and t - 1 is done with
      if (issued < T) issue(issued, (j + NBUF - 1) % NBUF), ++issued;
      const int k0 = (first + t * STEP) * kKeys;
      if (k0 < lim_hi) {
        const char* Kt = stages + j * STAGE;
        const char* Vt = Kt + kTile;
        bf16x8 kf[8], vf[4], pb[2];
#pragma unroll
        for (int s = 0; s < 8; ++s) kf[s] = row_frag(Kt, lane % 32, s, hh);
        f32x16 sc = f32x16{};
#pragma unroll
        for (int s = 0; s < 8; ++s) sc = mfma_bf16(kf[s], qf[s], sc);
        __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);  // DS reads
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // MFMA
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
#pragma unroll
        for (int w = 0; w < 4; ++w) vf[w] = v_frag(Vt, vo[w], 0);
        if (k0 + kKeys > lim_lo) {  // value k: key k0 + 8(k/4) + 4 hh + k%4 of this lane's row
          const int left = lim - k0 - 4 * hh;
#pragma unroll
          for (int k = 0; k < 16; ++k) sc[k] = 8 * (k / 4) + k % 4 < left ? sc[k] : -__builtin_inff();
        }
        float mx = sc[0];
#pragma unroll
        for (int k = 1; k < 16; ++k) mx = fmaxf(mx, sc[k]);
        mx = halves_max(mx) * c.scale_log2;
        if (__any(mx > m + kTau)) {
          const float mnew = fmaxf(m, mx), alpha = __builtin_amdgcn_exp2f(m - mnew);
          m = mnew;
          l *= alpha;
#pragma unroll
          for (int w = 0; w < 4; ++w) acc[w] *= alpha;
        }
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const float p = __builtin_amdgcn_exp2f(fmaf(sc[k], c.scale_log2, -m));
          sum[k % 2] += p;
          pb[k / 8][k % 8] = (bf16)p;
        }
        l += sum[0] + sum[1];
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          acc[w] = mfma_bf16(vf[w], pb[0], acc[w]);
          vf[w] = v_frag(Vt, vo[w], 1);
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) acc[w] = mfma_bf16(vf[w], pb[1], acc[w]);
        __builtin_amdgcn_s_setprio(0);
      }
      ++t;
    }
  }
  l = halves_sum(l);

  if constexpr (QW == 1) {  // join the four waves: lane = row, channels 32 w + 8 j + 4 hh + e
    __syncthreads();
    float* os = reinterpret_cast<float*>(lds);                  // [4][32][132]
    float2* ml = reinterpret_cast<float2*>(os + 4 * 32 * 132);  // [4][32]
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<float4*>(os + (wave * 32 + lane % 32) * 132 + 32 * w + 8 * j + 4 * hh) =
            make_float4(acc[w][4 * j], acc[w][4 * j + 1], acc[w][4 * j + 2], acc[w][4 * j + 3]);
    if (hh == 0) ml[wave * 32 + lane] = make_float2(m, l);
    __syncthreads();
    // thread: row tid / 8, channels 16 (tid % 8) ..
    const int row = threadIdx.x / 8, c0 = 16 * (threadIdx.x % 8), rr = row0 + row;
    if (rr >= a.R) return;
    float mx = kNoMax, sum = 0.f, o[16] = {};
#pragma unroll
    for (int w = 0; w < 4; ++w) mx = fmaxf(mx, ml[w * 32 + row].x);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float2 v = ml[w * 32 + row];
      const float f = __builtin_amdgcn_exp2f(v.x - mx);
      sum = fmaf(f, v.y, sum);
#pragma unroll
      for (int e = 0; e < 16; ++e) o[e] = fmaf(f, os[(w * 32 + row) * 132 + c0 + e], o[e]);
    }
    if (pt.left >= 0) {
      const long at = ((long)pt.left * pt.splits + pt.split) * 32 + row;
      store8(a.part + at * D + c0, o);
      store8(a.part + at * D + c0 + 8, o + 8);
      if (c0 == 0) a.ml[at] = make_float2(mx, sum);
      return;
    }
    const int ii = rr / c.G, gg = rr % c.G, head = pt.hk * c.G + gg;
    const float f = row_inverse(sum);
#pragma unroll
    for (int e = 0; e < 16; ++e) o[e] *= f;
    bf16* out = reinterpret_cast<bf16*>(c.O.p + pt.b * c.O.b + head * c.O.h + ii * c.O.n) + c0;
    store8(out, o);
    store8(out + 8, o + 8);
    if (a.lse && c0 == 0)
      a.lse[(pt.b * a.heads + head) * c.Nq + ii] = row_lse(mx, sum);
  } else {
    if (pt.left >= 0) {
      const long at = ((long)pt.left * pt.splits + pt.split) * 128 + wave * 32 + lane % 32;
      if (row0 + lane % 32 >= a.R) return;
      store_grad_row<false>(a.part + at * D, acc, 1.f, hh, nullptr, nullptr);
      if (hh == 0) a.ml[at] = make_float2(m, l);
      return;
    }
    __syncthreads();  // every wave is done with the stages
    rows_from_acc(lds + wave * 8192, acc, row_inverse(l), row_base(c.O, pt.b, pt.hk, c.G), row0, a.R, lane);
    int q = row0 + lane % 32;
    asm volatile("" : "+v"(q));  // (divided again here, or the first quotient stays in a register all the way)
    if (a.lse && hh == 0 && q < a.R)
      a.lse[(pt.b * a.heads + pt.hk * c.G + q % c.G) * c.Nq + q / c.G] = row_lse(m, l);
  }
}

// fp32: four waves of 16 rows each walk the keys in tiles of 32 staged in LDS.
template <int D>
__global__ __launch_bounds__(256, D == 64 ? 1 : 3) void attn_f32x_kernel(const FwdArgs a) {
  constexpr int W = D / 16, LD = D + 4, PT = 32 * D / 4 / 256;  // 16-byte pieces per thread, tensor and tile
  __shared__ __attribute__((aligned(16))) float ks[32 * LD], vs[32 * LD];
  const AttnCall& c = a.c;
  const Part pt = part_of(a.cut, c.Hkv, blockIdx.x);
  const int wave = wave_uniform(threadIdx.x / 64), lane = threadIdx.x % 64, gr = lane / 16;
  const int n = attn_keys(c, pt.b);
  const int row0 = pt.tile * 64 + wave * 16;
  const int r = min(row0 + lane % 16, a.R - 1), i = r / c.G, g = r % c.G;
  const int lim = attn_limit(c, n, i);
  const int lim_lo = attn_limit(c, n, min(row0, a.R - 1) / c.G);
  const int lim_hi = row0 < a.R ? attn_limit(c, n, min(row0 + 15, a.R - 1) / c.G) : 0;
  const int end = max(0, attn_limit(c, n, min(pt.tile * 64 + 63, a.R - 1) / c.G));
  const int all = (end + 31) / 32, per = (all + pt.splits - 1) / pt.splits;
  const int t0 = pt.split * per, t1 = min(all, t0 + per);
  const char* Kh = c.K.p + pt.b * c.K.b + pt.hk * c.K.h;
  const char* Vh = c.V.p + pt.b * c.V.b + pt.hk * c.V.h;
  float4 qv[W];
  f32_quarter<D>(c.Q.p + pt.b * c.Q.b + (pt.hk * c.G + g) * c.Q.h + i * c.Q.n, lane, qv);
  f32x4 acc[W];
#pragma unroll
  for (int w = 0; w < W; ++w) acc[w] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = kNoMax, l = 0.f;
  float4 kn[PT], vn[PT];
  auto fetch = [&](int t) {
#pragma unroll
    for (int x = 0; x < PT; ++x) {
      const int e = threadIdx.x + 256 * x, row = e / (D / 4), at = e % (D / 4);
      const long key = min(t * 32 + row, n - 1);
      kn[x] = reinterpret_cast<const float4*>(Kh + key * c.K.n)[at];
      vn[x] = reinterpret_cast<const float4*>(Vh + key * c.V.n)[at];
    }
  };
  if (t0 < t1) fetch(t0);
  for (int t = t0; t < t1; ++t) {
    __syncthreads();
#pragma unroll
    for (int x = 0; x < PT; ++x) {
      const int e = threadIdx.x + 256 * x, row = e / (D / 4), at = e % (D / 4);
      *reinterpret_cast<float4*>(ks + row * LD + 4 * at) = kn[x];
      *reinterpret_cast<float4*>(vs + row * LD + 4 * at) = vn[x];
    }
    __syncthreads();
    if (t + 1 < t1) fetch(t + 1);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int k0 = t * 32 + 16 * u;
      if (k0 >= lim_hi) break;
      const f32x4 sc = f32_rows<D>(ks + 16 * u * LD, qv, lane);
      float p[4], mx = -__builtin_inff();
#pragma unroll
      for (int k = 0; k < 4; ++k) {  // key k0 + 4 gr + k
        p[k] = sc[k] * c.scale_log2;
        if (k0 + 16 > lim_lo) p[k] = k0 + 4 * gr + k < lim ? p[k] : -__builtin_inff();
        mx = fmaxf(mx, p[k]);
      }
      const float mnew = fmaxf(m, rows_max(mx)), alpha = __builtin_amdgcn_exp2f(m - mnew);
      m = mnew;
      l *= alpha;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        p[k] = __builtin_amdgcn_exp2f(p[k] - mnew);
        l += p[k];
      }
#pragma unroll
      for (int w = 0; w < W; ++w) acc[w] *= alpha;
      f32_cols<D>(vs + 16 * u * LD, p, acc, lane);
    }
  }
  l = rows_sum(l);
  if (row0 + lane % 16 >= a.R) return;
  if (pt.left >= 0) {
    const long at = ((long)pt.left * pt.splits + pt.split) * 64 + wave * 16 + lane % 16;
    f32_store<D>(reinterpret_cast<char*>(a.part + at * D), acc, 1.f, lane);
    if (gr == 0) a.ml[at] = make_float2(m, l);
    return;
  }
  const int head = pt.hk * c.G + g;
  f32_store<D>(c.O.p + pt.b * c.O.b + head * c.O.h + i * c.O.n, acc, row_inverse(l), lane);
  if (a.lse && gr == 0)
    a.lse[(pt.b * a.heads + head) * c.Nq + i] = row_lse(m, l);
}

// fp32, few rows: a workgroup has 16 of them and its four waves take every fourth sub-tile of 16 keys, straight
// from memory; they add up through LDS.
template <int D>
__global__ __launch_bounds__(256, D == 64 ? 1 : 2) void attn_f32_few_kernel(const FwdArgs a) {
  constexpr int W = D / 16;
  __shared__ __attribute__((aligned(16))) float os[4 * 16 * (D + 4)];
  __shared__ float2 mls[4][16];
  const AttnCall& c = a.c;
  const Part pt = part_of(a.cut, c.Hkv, blockIdx.x);
  const int wave = wave_uniform(threadIdx.x / 64), lane = threadIdx.x % 64, gr = lane / 16;
  const int n = attn_keys(c, pt.b), row0 = pt.tile * 16;
  const int r = min(row0 + lane % 16, a.R - 1), i = r / c.G, g = r % c.G;
  const int lim = attn_limit(c, n, i);
  const int end = max(0, attn_limit(c, n, min(row0 + 15, a.R - 1) / c.G));
  const int all = (end + 15) / 16, per = (all + pt.splits - 1) / pt.splits;
  const int t0 = pt.split * per, t1 = min(all, t0 + per);
  const char* Kh = c.K.p + pt.b * c.K.b + pt.hk * c.K.h;
  const char* Vh = c.V.p + pt.b * c.V.b + pt.hk * c.V.h;
  float4 qv[W], kv[W], vv[4][D / 64];
  f32_quarter<D>(c.Q.p + pt.b * c.Q.b + (pt.hk * c.G + g) * c.Q.h + i * c.Q.n, lane, qv);
  f32x4 acc[W];
#pragma unroll
  for (int w = 0; w < W; ++w) acc[w] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = kNoMax, l = 0.f;
  auto keys = [&](int t) { f32_quarter<D>(Kh + min(t * 16 + lane % 16, n - 1) * c.K.n, lane, kv); };
  auto values = [&](int t) { f32_pieces<D>(Vh, c.V.n, t * 16, n - 1, lane, vv); };
  if (t0 + wave < t1) {
    keys(t0 + wave);
    values(t0 + wave);
  }
  for (int t = t0 + wave; t < t1; t += 4) {
    const int nxt = min(t + 4, t1 - 1);
    const f32x4 sc = f32_rows<D>(kv, qv);
    keys(nxt);
    float p[4], mx = -__builtin_inff();
#pragma unroll
    for (int k = 0; k < 4; ++k) {  // key 16 t + 4 gr + k
      p[k] = 16 * t + 4 * gr + k < lim ? sc[k] * c.scale_log2 : -__builtin_inff();
      mx = fmaxf(mx, p[k]);
    }
    const float mnew = fmaxf(m, rows_max(mx)), alpha = __builtin_amdgcn_exp2f(m - mnew);
    m = mnew;
    l *= alpha;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      p[k] = __builtin_amdgcn_exp2f(p[k] - mnew);
      l += p[k];
    }
#pragma unroll
    for (int w = 0; w < W; ++w) acc[w] *= alpha;
    f32_cols<D>(vv, p, acc);
    values(nxt);
  }
  l = rows_sum(l);
  if (gr == 0) mls[wave][lane] = make_float2(m, l);
  __syncthreads();
  float mx = kNoMax, sum = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) mx = fmaxf(mx, mls[w][lane % 16].x);
  const float f = __builtin_amdgcn_exp2f(m - mx);
#pragma unroll
  for (int w = 0; w < W; ++w) acc[w] *= f;
  float o[W];
  f32_join<D>(os, acc, wave, lane, o);
  const int row = threadIdx.x / 16, rr = row0 + row, c0 = (threadIdx.x % 16) * W;
  if (rr >= a.R) return;
  mx = kNoMax;
#pragma unroll
  for (int w = 0; w < 4; ++w) mx = fmaxf(mx, mls[w][row].x);
#pragma unroll
  for (int w = 0; w < 4; ++w) sum = fmaf(__builtin_amdgcn_exp2f(mls[w][row].x - mx), mls[w][row].y, sum);
  const int ii = rr / c.G, head = pt.hk * c.G + rr % c.G;
  const long at = ((long)pt.left * pt.splits + pt.split) * 16 + row;
  const float inv = pt.left >= 0 ? 1.f : row_inverse(sum);
  float* out = pt.left >= 0 ? a.part + at * D
                            : reinterpret_cast<float*>(c.O.p + pt.b * c.O.b + head * c.O.h + ii * c.O.n);
#pragma unroll
  for (int s = 0; s < W / 4; ++s)
    reinterpret_cast<float4*>(out + c0)[s] =
        make_float4(o[4 * s] * inv, o[4 * s + 1] * inv, o[4 * s + 2] * inv, o[4 * s + 3] * inv);
  if (c0 != 0) return;
  if (pt.left >= 0)
    a.ml[at] = make_float2(mx, sum);
  else if (a.lse)
    a.lse[(pt.b * a.heads + head) * c.Nq + ii] = row_lse(mx, sum);
}

// Joins the parts of a cut tile's rows: a wave per row, D / 64 channels per lane.
template <typename T, int D>
__global__ __launch_bounds__(256) void attn_join_kernel(const FwdArgs a) {
  constexpr int V = D / 64;
  const AttnCall& c = a.c;
  const long at = (long)blockIdx.x * 4 + threadIdx.x / 64;  // (cut tile, row): rows is a multiple of 4
  const int lane = threadIdx.x % 64, S = a.cut.splits;
  const long left = at / a.rows;
  const int row = (int)(at % a.rows);
  int tile;
  long bh;
  cut_tile(a.cut, a.cut.whole + (int)left, &tile, &bh);
  const int r = tile * a.rows + row;
  if (r >= a.R) return;
  // lane s: the weight of part s (at most 64); then the parts' rows, eight in flight
  const float2 v = lane < S ? a.ml[(left * S + lane) * a.rows + row] : make_float2(kNoMax, 0.f);
  const float* part = a.part + (left * S * a.rows + row) * D + lane * V;
  float mx = rows_max(v.x);
#pragma unroll
  for (int d = 8; d >= 1; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
  const float f = __builtin_amdgcn_exp2f(v.x - mx);
  float sum = rows_sum(f * v.y);
#pragma unroll
  for (int d = 8; d >= 1; d >>= 1) sum += __shfl_xor(sum, d);
  float o[V] = {};
  for (int s0 = 0; s0 < S; s0 += 8) {
    float x[8][V];
#pragma unroll
    for (int u = 0; u < 8; ++u)
#pragma unroll
      for (int k = 0; k < V; ++k) x[u][k] = part[(long)min(s0 + u, S - 1) * a.rows * D + k];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float w = s0 + u < S ? __shfl(f, s0 + u) : 0.f;
#pragma unroll
      for (int k = 0; k < V; ++k) o[k] = fmaf(w, x[u][k], o[k]);
    }
  }
  const int b = (int)(bh / c.Hkv), i = r / c.G, head = (int)(bh % c.Hkv) * c.G + r % c.G;
  const float inv = row_inverse(sum);
  T* out = reinterpret_cast<T*>(c.O.p + b * c.O.b + head * c.O.h + i * c.O.n) + lane * V;
#pragma unroll
  for (int k = 0; k < V; ++k) out[k] = from_f32<T>(o[k] * inv);
  if (a.lse && lane == 0)
    a.lse[(b * a.heads + head) * c.Nq + i] = row_lse(mx, sum);
}

// How a call is cut: rows per tile, and the parts of the tiles.
struct FwdPlan {
  int rows;
  Cut cut;
};
FwdPlan fwd_plan(const AttnShape& s) {
  const int R = s.Nq * (s.H / s.Hkv), bh = s.B * s.Hkv, steps = (s.Nk + 31) / 32;
  // few rows. bf16: bound by reading K and V, in parts of a quarter round; fp32: by latency
  const bool few = s.bf16 ? R <= 32 : f32_few((R + 63) / 64, bh) && (s.d == 64 || attn_work(s) < kFewForward);
  const int rows = few ? (s.bf16 ? 32 : 16) : s.bf16 ? 128 : 64, tiles = (R + rows - 1) / rows;
  const double bytes = rows * (s.d + 2) * 4.0;
  if (few && s.bf16) return {rows, make_cut(tiles, bh, false, 4 * kCus, steps, 0.4, bytes, 16)};
  if (few) return {rows, make_cut(tiles, bh, s.causal, 4 * kCus, (s.Nk + 63) / 64, 1.5, bytes, 2)};
  return {rows, make_cut(tiles, bh, s.causal, s.bf16 ? 3 * kCus : 4 * kCus, steps, s.bf16 ? 0.9 : 2.0, bytes, 8)};
}

}  // namespace

size_t attn_workspace_bytes(const AttnShape& s) {
  const FwdPlan p = fwd_plan(s);
  return (size_t)cut_left(p.cut) * p.cut.splits * p.rows * (s.d + 2) * sizeof(float);
}

hipError_t launch_attn(const AttnShape& s, const HeadView& Q, const HeadView& K, const HeadView& V,
                       const int32_t* kv_len, float scale, const HeadView& O, float* lse, void* ws,
                       hipStream_t st) {
  const FwdPlan p = fwd_plan(s);
  FwdArgs a{};
  a.c = attn_call(s, Q, K, V, O, kv_len, scale);
  a.cut = p.cut;
  a.R = s.Nq * (s.H / s.Hkv);
  a.rows = p.rows;
  a.heads = s.H;
  a.lse = lse;
  const long parts = cut_left(p.cut) * p.cut.splits * p.rows;  // rows of partial sums
  a.part = (float*)ws;
  a.ml = (float2*)((float*)ws + parts * s.d);
  const auto kernel = s.bf16         ? (p.rows == 32 ? attn_bf16_kernel<1> : attn_bf16_kernel<4>)
                      : p.rows == 16 ? (s.d == 64 ? attn_f32_few_kernel<64> : attn_f32_few_kernel<128>)
                                     : (s.d == 64 ? attn_f32x_kernel<64> : attn_f32x_kernel<128>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)p.cut.total), dim3(256), 0, st, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || parts == 0) return e;
  const auto join = s.bf16 ? attn_join_kernel<bf16, 128>
                           : s.d == 64 ? attn_join_kernel<float, 64> : attn_join_kernel<float, 128>;
  hipLaunchKernelGGL(join, dim3((unsigned)(cut_left(p.cut) * p.rows / 4)), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace rola
