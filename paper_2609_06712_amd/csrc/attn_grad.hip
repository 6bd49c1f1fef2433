// Gradients of the softmax attention of attn.hip (attn_common.h): from dO, O and the forward's log-sum-exp,
//   P = exp2(S scale log2e - lse),  D = rowsum(dO O),  dP = dO V^T,  dS = P (dP - D),
//   dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO  (dK, dV summed over the query heads of a key head).
// The probabilities are recomputed, twice, so that every gradient is summed in registers in a fixed order
// and is rounded once: a pass over the keys per tile of rows (dQ, three products; four in bf16, whose dS is two
// terms) and a pass over the queries per block of keys (dK, dV, four). Bound by the matrix cores: 14 d operations
// per visible pair (bf16, with the pass for D: 20 d) against the ten of a single pass, which would have to add dQ in
// memory. Measured in a kernel trace, bf16, 8400 x 8400, 12 heads: D 355 us (1.22 PFLOP/s), dQ 761 (1.14), dK and dV
// 909 (0.95); matrix cores busy 0.77, 0.69 and 0.52 of the cycles.
//
// D. It is rowsum(dO O), but from an O that was rounded to bf16 it is off by dO times that rounding, for all
// keys of a row alike: sum_j P_ij K_j times the error reaches dQ, where sum_j dS_ij K_j has cancelled (8400 keys:
// dQ off by 0.0048 of its norm, where its own rounding is 0.0017). So bf16 sums it in fp32 from what the
// gradients use, D = rowsum(P dP), in a pass of two products (attn_rowsum_bf16_kernel); fp32 takes dO O.
//
// Row statistics: per query lse (bf16: less kLift) and D, in tiles of 32 queries [32 lse][32 D], per head padded to
// whole tiles with lse = inf: P is then zero for rows past the last and for rows that see no key, with no test in the
// walk.
//
// The tiles that do not fill a round of the chip are cut (Cut); the parts' fp32 sums go to the workspace and are
// added in order by attn_sum_kernel.
#include <algorithm>

#include "attn_common.h"

namespace rola {
namespace {

constexpr int kRows = 32;            // rows of a sub-tile
constexpr int kTile = kRows * 256;   // its bytes (bf16, d 128)
// The bf16 dK/dV pass works with 2^15 P: one role hands it to the other as fp16, whose normal range starts at 2^-14, and
// many keys, or one that takes nearly all of a row, leave the others less. Lifted, P fills that range up to its end (32768
// of 65504) and is rounded by half a step of fp16 from 2^-29 on. Without it P below 2^-25 gave dK = 0, dK of 300000
// keys was off by 0.0039 of its norm (0.0024), and single keys beside one that takes 0.999 of 8400 by up to 0.064 of
// theirs (0.0049). The factor is a power of two, so no other rounding changes but that of lse - 15, 2^-21 at most below
// an lse of 31; the times do not change. dK and dV are summed at 2^15 times their size, so what exceeds 2^112 comes out
// infinite.
constexpr float kLift = 15.f, kDrop = 1.f / 32768;
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t pair_bf16(float a, float b) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, bf16x2{(bf16)a, (bf16)b});
}
__device__ __forceinline__ uint32_t pair_f16(float a, float b) {
  return __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b});
}

struct GradArgs {
  AttnCall c;     // c.O: dO
  View G1, G2;    // dQ; or dK, dV
  Cut cut;
  int R, Np, H;
  const float* stat;   // [B, H, Np / 32][lse, D][32]
  const float* lse;    // [B, H, Nq], the forward's
  float* dsum;         // attn_rowsum_bf16_kernel: D of the whole tiles' rows [B Hkv][R]
  float* part;         // sums of the cut tiles: [left][splits][rows of a tile][d] (D: without d), dV's after dK's
  long part2;          // elements between dK's and dV's
};

// Where the statistics of query i of a head are: lse there, D 32 further.
__device__ __forceinline__ long stat_at(long head, int Np, int i) { return (head * (Np / 32) + i / 32) * 64 + i % 32; }

// lse, less kLift, and D (of a cut tile the sum of its parts) into tiles; queries as rows i G + g of their key head.
__global__ __launch_bounds__(256) void attn_stat_kernel(const GradArgs a, long rows, float* __restrict__ stat) {
  const long row = (long)blockIdx.x * 256 + threadIdx.x;  // (b, h, padded query)
  if (row >= rows) return;
  const int G = a.c.G, S = a.cut.splits;
  const long head = row / a.Np, bh = head / G;
  const int i = (int)(row % a.Np);
  float l = -__builtin_inff(), s = 0.f;
  if (i < a.c.Nq) {
    l = a.lse[head * a.c.Nq + i];
    const int r = i * G + (int)(head % G), place = cut_place(a.cut, r / 256, bh);
    if (place < a.cut.whole) {
      s = a.dsum[bh * a.R + r];
    } else {
      const float* p = a.part + (long)(place - a.cut.whole) * S * 256 + r % 256;
      for (int k = 0; k < S; ++k) s += p[k * 256];
    }
  }
  const bool none = saw_no_key(l);
  float* at = stat + stat_at(head, a.Np, i);
  at[0] = none ? __builtin_inff() : l - kLift;
  at[32] = none ? 0.f : s;
}

// A workgroup takes every gridDim.x-th set of 16 rows: one set each would be a grid of more than 2^32 threads from 2^28
// rows on, which cannot be launched.
constexpr int kRowdotGrid = 1 << 16;
__global__ __launch_bounds__(256) void attn_rowdot_f32_kernel(int H, int Nq, int Np, int d, long rows, View O,
                                                              View dO, const float* __restrict__ lse,
                                                              float* __restrict__ stat) {
  const int part = threadIdx.x % 16;
  for (long row = (long)blockIdx.x * 16 + threadIdx.x / 16; row < rows; row += (long)gridDim.x * 16) {
    const long bh = row / Np;
    const int i = (int)(row % Np), b = (int)(bh / H), h = (int)(bh % H);
    float s = 0.f;
    if (i < Nq) {
      const float4* x = reinterpret_cast<const float4*>(O.p + b * O.b + h * O.h + i * O.n);
      const float4* y = reinterpret_cast<const float4*>(dO.p + b * dO.b + h * dO.h + i * dO.n);
      for (int e = part; e < d / 4; e += 16) {
        const float4 u = x[e], v = y[e];
        s = fmaf(u.x, v.x, fmaf(u.y, v.y, fmaf(u.z, v.z, fmaf(u.w, v.w, s))));
      }
    }
#pragma unroll
    for (int off = 8; off >= 1; off >>= 1) s += __shfl_xor(s, off, 16);
    if (part == 0) {
      const float l = i < Nq ? lse[bh * Nq + i] : -__builtin_inff();
      const bool none = saw_no_key(l);
      float* at = stat + stat_at(bh, Np, i);
      at[0] = none ? __builtin_inff() : l;
      at[32] = none ? 0.f : s;
    }
  }
}

// ---- dQ ------------------------------------------------------------------------------------------------

// D = rowsum(P dP): four waves of 64 rows walk the keys in sub-tiles of 32 through three LDS stages. Two row
// tiles per wave: an operand read from LDS serves two products, and without a gradient's accumulators two
// workgroups fit a CU.
__global__ __launch_bounds__(256, 2) void attn_rowsum_bf16_kernel(const GradArgs a) {
  constexpr int STAGE = 2 * kTile, NBUF = 3, DPW = 2;
  __shared__ __attribute__((aligned(1024))) char lds[NBUF * STAGE];
  const AttnCall& c = a.c;
  const Part pt = part_of(a.cut, c.Hkv, blockIdx.x);
  const int wave = wave_uniform(threadIdx.x / 64), lane = threadIdx.x % 64, hh = lane / 32;
  const int n = attn_keys(c, pt.b);
  const int row0 = (pt.tile * 4 + wave) * 64;
  const int lim_lo = attn_limit(c, n, min(row0, a.R - 1) / c.G);
  const int lim_hi = row0 < a.R ? attn_limit(c, n, min(row0 + 63, a.R - 1) / c.G) : 0;
  const int end = max(0, attn_limit(c, n, min(pt.tile * 256 + 255, a.R - 1) / c.G));
  const int all = (end + 31) / 32, per = (all + pt.splits - 1) / pt.splits;
  const int first = pt.split * per, T = max(0, min(all, first + per) - first);
  const char* Kh = c.K.p + pt.b * c.K.b + pt.hk * c.K.h;
  const char* Vh = c.V.p + pt.b * c.V.b + pt.hk * c.V.h;
  uint32_t dk[DPW], dv[DPW];
#pragma unroll
  for (int x = 0; x < DPW; ++x) {
    const int row = 4 * (wave * DPW + x) + lane / 16;
    const uint32_t chunk = ((lane % 16) ^ bw_swizzle(row)) << 4;
    dk[x] = row * (uint32_t)c.K.n + chunk;
    dv[x] = row * (uint32_t)c.V.n + chunk;
  }
  const uint32_t lds0 = lds_address(lds) + wave * DPW * 1024;
  bf16x8 qf[2][8], df[2][8];
  int lim[2];
  float lse[2], sum[2] = {0.f, 0.f};
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int r = min(row0 + 32 * u + lane % 32, a.R - 1), i = r / c.G, head = pt.hk * c.G + r % c.G;
    lim[u] = attn_limit(c, n, i);
    const char* q = c.Q.p + pt.b * c.Q.b + head * c.Q.h + i * c.Q.n + 16 * hh;
    const char* o = c.O.p + pt.b * c.O.b + head * c.O.h + i * c.O.n + 16 * hh;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      qf[u][s] = *reinterpret_cast<const bf16x8*>(q + 32 * s);
      df[u][s] = *reinterpret_cast<const bf16x8*>(o + 32 * s);
    }
    lse[u] = a.lse[((long)pt.b * a.H + head) * c.Nq + i];
    if (saw_no_key(lse[u])) lse[u] = __builtin_inff();
  }
  wait_vm<0>();

  auto issue = [&](int t, int buf) {
    const int k0 = (first + t) * 32;
    const uint32_t dst = lds0 + buf * STAGE;
    const char* kb = Kh + (long)k0 * c.K.n;
    const char* vb = Vh + (long)k0 * c.V.n;
#pragma unroll
    for (int x = 0; x < DPW; ++x) {
      uint32_t ok = dk[x], ov = dv[x];
      if (k0 + 32 > n) {  // rows past the last key re-read it
        const int back = max(4 * (wave * DPW + x) + lane / 16 - (n - 1 - k0), 0);
        ok -= back * (uint32_t)c.K.n;
        ov -= back * (uint32_t)c.V.n;
      }
      dma16(kb, ok, dst + x * 1024);
      dma16(vb, ov, dst + kTile + x * 1024);
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
      if (issued == t + NBUF - 1)
        wait_vm<2 * DPW * (NBUF - 2)>();
      else
        __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
      if (issued < T) issue(issued, (j + NBUF - 1) % NBUF), ++issued;
      const int k0 = (first + t) * 32;
      if (k0 < lim_hi) {
        const char* Kt = lds + j * STAGE;
        f32x16 sc[2] = {f32x16{}, f32x16{}}, dp[2] = {f32x16{}, f32x16{}};
#pragma unroll
        for (int s = 0; s < 8; ++s) {
          const bf16x8 x = row_frag(Kt, lane % 32, s, hh), y = row_frag(Kt + kTile, lane % 32, s, hh);
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            sc[u] = mfma_bf16(x, qf[u][s], sc[u]);
            dp[u] = mfma_bf16(y, df[u][s], dp[u]);
          }
        }
        __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);  // DS reads
#pragma unroll
        for (int s = 0; s < 10; ++s) {
          __builtin_amdgcn_sched_group_barrier(0x008, 2, 0);  // MFMA
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        if (k0 + 32 > lim_lo) {  // value k: key k0 + 8(k/4) + 4 hh + k%4 of this lane's rows
#pragma unroll
          for (int u = 0; u < 2; ++u) {
            const int left = lim[u] - k0 - 4 * hh;
#pragma unroll
            for (int k = 0; k < 16; ++k) sc[u][k] = 8 * (k / 4) + k % 4 < left ? sc[u][k] : -__builtin_inff();
          }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int k = 0; k < 16; ++k)
            sum[u] = fmaf(__builtin_amdgcn_exp2f(fmaf(sc[u][k], c.scale_log2, -lse[u])), dp[u][k], sum[u]);
      }
      ++t;
    }
  }
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int r = row0 + 32 * u + lane % 32;
    const float s = halves_sum(sum[u]);
    if (r >= a.R || hh != 0) continue;
    if (pt.left >= 0)
      a.part[((long)pt.left * pt.splits + pt.split) * 256 + wave * 64 + 32 * u + lane] = s;
    else
      a.dsum[pt.bh * a.R + r] = s;
  }
}

// Four waves of 32 rows walk the keys in sub-tiles of 32 through three LDS stages:
//   S^T = K Q^T, dP^T = V dO^T (a lane has one row and 16 keys of it), dQ^T += K^T dS^T.
// dS goes into its product as two bf16 terms, the rounded value and what that left: the sum over the keys
// cancels, and one term's rounding alone would be 0.0019 to 0.0021 of dQ's norm beside dQ's own 0.0017.
__global__ __launch_bounds__(256, 2) void attn_dq_bf16_kernel(const GradArgs a) {
  constexpr int STAGE = 2 * kTile, NBUF = 3, DPW = 2;
  __shared__ __attribute__((aligned(1024))) char lds[NBUF * STAGE];
  const AttnCall& c = a.c;
  const Part pt = part_of(a.cut, c.Hkv, blockIdx.x);
  const int wave = wave_uniform(threadIdx.x / 64), lane = threadIdx.x % 64, hh = lane / 32;
  const int n = attn_keys(c, pt.b);
  const int row0 = (pt.tile * 4 + wave) * 32;
  const int r = min(row0 + lane % 32, a.R - 1), i = r / c.G, head = pt.hk * c.G + r % c.G;
  const int lim = attn_limit(c, n, i);
  const int lim_lo = attn_limit(c, n, min(row0, a.R - 1) / c.G);
  const int lim_hi = row0 < a.R ? attn_limit(c, n, min(row0 + 31, a.R - 1) / c.G) : 0;
  const int end = max(0, attn_limit(c, n, min(pt.tile * 128 + 127, a.R - 1) / c.G));
  const int all = (end + 31) / 32, per = (all + pt.splits - 1) / pt.splits;
  const int first = pt.split * per, T = max(0, min(all, first + per) - first);
  const char* Kh = c.K.p + pt.b * c.K.b + pt.hk * c.K.h;
  const char* Vh = c.V.p + pt.b * c.V.b + pt.hk * c.V.h;
  uint32_t dk[DPW], dv[DPW];
#pragma unroll
  for (int x = 0; x < DPW; ++x) {
    const int row = 4 * (wave * DPW + x) + lane / 16;
    const uint32_t chunk = ((lane % 16) ^ bw_swizzle(row)) << 4;
    dk[x] = row * (uint32_t)c.K.n + chunk;
    dv[x] = row * (uint32_t)c.V.n + chunk;
  }
  const uint32_t lds0 = lds_address(lds) + wave * DPW * 1024;
  bf16x8 qf[8], df[8];
  {
    const char* q = c.Q.p + pt.b * c.Q.b + head * c.Q.h + i * c.Q.n + 16 * hh;
    const char* o = c.O.p + pt.b * c.O.b + head * c.O.h + i * c.O.n + 16 * hh;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      qf[s] = *reinterpret_cast<const bf16x8*>(q + 32 * s);
      df[s] = *reinterpret_cast<const bf16x8*>(o + 32 * s);
    }
  }
  float lse = a.lse[((long)pt.b * a.H + head) * c.Nq + i];
  if (saw_no_key(lse)) lse = __builtin_inff();
  const float dsum = a.stat[stat_at((long)pt.b * a.H + head, a.Np, i) + 32];
  wait_vm<0>();
  f32x16 acc[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) acc[w] = f32x16{};

  auto issue = [&](int t, int buf) {
    const int k0 = (first + t) * 32;
    const uint32_t dst = lds0 + buf * STAGE;
    const char* kb = Kh + (long)k0 * c.K.n;
    const char* vb = Vh + (long)k0 * c.V.n;
#pragma unroll
    for (int x = 0; x < DPW; ++x) {
      uint32_t ok = dk[x], ov = dv[x];
      if (k0 + 32 > n) {  // rows past the last key re-read it
        const int back = max(4 * (wave * DPW + x) + lane / 16 - (n - 1 - k0), 0);
        ok -= back * (uint32_t)c.K.n;
        ov -= back * (uint32_t)c.V.n;
      }
      dma16(kb, ok, dst + x * 1024);
      dma16(vb, ov, dst + kTile + x * 1024);
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
      if (issued == t + NBUF - 1)
        wait_vm<2 * DPW * (NBUF - 2)>();
      else
        __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
      if (issued < T) issue(issued, (j + NBUF - 1) % NBUF), ++issued;
      const int k0 = (first + t) * 32;
      if (k0 < lim_hi) {
        const char* Kt = lds + j * STAGE;
        const char* Vt = Kt + kTile;
        bf16x8 ka[8], va[8], kt[8];
        f32x16 sc = f32x16{}, dp = f32x16{};
        __builtin_amdgcn_s_setprio(0);
#pragma unroll
        for (int s = 0; s < 8; ++s) {
          ka[s] = row_frag(Kt, lane % 32, s, hh);
          va[s] = row_frag(Vt, lane % 32, s, hh);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int w = 0; w < 4; ++w) kt[4 * u + w] = tr_frag(Kt, w, u, lane);
#pragma unroll
        for (int s = 0; s < 8; ++s) {
          sc = mfma_bf16(ka[s], qf[s], sc);
          dp = mfma_bf16(va[s], df[s], dp);
        }
        __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);  // DS reads
#pragma unroll
        for (int s = 0; s < 16; ++s) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // MFMA
          __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        }
        if (k0 + 32 > lim_lo) {  // value k: key k0 + 8(k/4) + 4 hh + k%4 of this lane's row
          const int left = lim - k0 - 4 * hh;
#pragma unroll
          for (int k = 0; k < 16; ++k) sc[k] = 8 * (k / 4) + k % 4 < left ? sc[k] : -__builtin_inff();
        }
        __builtin_amdgcn_sched_barrier(0);
        // ahead of the other workgroup's scores: 8400 tokens, 12 heads 763 -> 735 us
        __builtin_amdgcn_s_setprio(1);
        bf16x8 ds[2], dl[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float p = __builtin_amdgcn_exp2f(fmaf(sc[8 * u + k], c.scale_log2, -lse));
            const float x = p * (dp[8 * u + k] - dsum);
            ds[u][k] = (bf16)x;
            dl[u][k] = (bf16)(x - (float)ds[u][k]);
          }
#pragma unroll
          for (int w = 0; w < 4; ++w) acc[w] = mfma_bf16(kt[4 * u + w], ds[u], acc[w]);
#pragma unroll
          for (int w = 0; w < 4; ++w) acc[w] = mfma_bf16(kt[4 * u + w], dl[u], acc[w]);
        }
        __builtin_amdgcn_sched_group_barrier(0x402, 60, 0);
#pragma unroll
        for (int s = 0; s < 8; ++s) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x402, 8, 0);
        }
      }
      ++t;
    }
  }
  if (pt.left >= 0) {
    if (row0 + lane % 32 < a.R)
      store_grad_row<false>(a.part + (((long)pt.left * pt.splits + pt.split) * 128 + wave * 32 + lane % 32) * 128, acc,
                            c.scale, hh, nullptr, nullptr);
    return;
  }
  __syncthreads();  // every wave is done with the stages
  rows_from_acc(lds + wave * 8192, acc, c.scale, row_base(a.G1, pt.b, pt.hk, c.G), row0, a.R, lane);
}

// fp32: four waves of 16 rows, key tiles of 32 staged in LDS.
template <int D>
__global__ __launch_bounds__(256, D == 64 ? 1 : 3) void attn_dq_f32_kernel(const GradArgs a) {
  constexpr int W = D / 16, LD = D + 4, PT = 32 * D / 4 / 256;
  __shared__ __attribute__((aligned(16))) float ks[32 * LD], vs[32 * LD];
  const AttnCall& c = a.c;
  const Part pt = part_of(a.cut, c.Hkv, blockIdx.x);
  const int wave = wave_uniform(threadIdx.x / 64), lane = threadIdx.x % 64, gr = lane / 16;
  const int n = attn_keys(c, pt.b);
  const int row0 = pt.tile * 64 + wave * 16;
  const int r = min(row0 + lane % 16, a.R - 1), i = r / c.G, head = pt.hk * c.G + r % c.G;
  const int lim = attn_limit(c, n, i);
  const int lim_hi = row0 < a.R ? attn_limit(c, n, min(row0 + 15, a.R - 1) / c.G) : 0;
  const int end = max(0, attn_limit(c, n, min(pt.tile * 64 + 63, a.R - 1) / c.G));
  const int all = (end + 31) / 32, per = (all + pt.splits - 1) / pt.splits;
  const int t0 = pt.split * per, t1 = min(all, t0 + per);
  const char* Kh = c.K.p + pt.b * c.K.b + pt.hk * c.K.h;
  const char* Vh = c.V.p + pt.b * c.V.b + pt.hk * c.V.h;
  float4 qv[W], dv[W];
  f32_quarter<D>(c.Q.p + pt.b * c.Q.b + head * c.Q.h + i * c.Q.n, lane, qv);
  f32_quarter<D>(c.O.p + pt.b * c.O.b + head * c.O.h + i * c.O.n, lane, dv);
  const float* st = a.stat + stat_at((long)pt.b * a.H + head, a.Np, i);
  const float lse = st[0], dsum = st[32];
  f32x4 acc[W];
#pragma unroll
  for (int w = 0; w < W; ++w) acc[w] = f32x4{0.f, 0.f, 0.f, 0.f};
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
      const f32x4 dp = f32_rows<D>(vs + 16 * u * LD, dv, lane);
      float ds[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float p = k0 + 4 * gr + k < lim ? __builtin_amdgcn_exp2f(fmaf(sc[k], c.scale_log2, -lse)) : 0.f;
        ds[k] = p * (dp[k] - dsum);
      }
      f32_cols<D>(ks + 16 * u * LD, ds, acc, lane);
    }
  }
  if (row0 + lane % 16 >= a.R) return;
  char* out = pt.left >= 0
                  ? reinterpret_cast<char*>(a.part + (((long)pt.left * pt.splits + pt.split) * 64 + wave * 16 + lane % 16) * D)
                  : a.G1.p + pt.b * a.G1.b + head * a.G1.h + i * a.G1.n;
  f32_store<D>(out, acc, c.scale, lane);
}

// fp32, few rows: 16 per workgroup, every fourth sub-tile of 16 keys per wave, straight from memory.
template <int D>
__global__ __launch_bounds__(256, D == 64 ? 1 : 2) void attn_dq_f32_few_kernel(const GradArgs a) {
  constexpr int W = D / 16;
  __shared__ __attribute__((aligned(16))) float os[4 * 16 * (D + 4)];
  const AttnCall& c = a.c;
  const Part pt = part_of(a.cut, c.Hkv, blockIdx.x);
  const int wave = wave_uniform(threadIdx.x / 64), lane = threadIdx.x % 64, gr = lane / 16;
  const int n = attn_keys(c, pt.b), row0 = pt.tile * 16;
  const int r = min(row0 + lane % 16, a.R - 1), i = r / c.G, head = pt.hk * c.G + r % c.G;
  const int lim = attn_limit(c, n, i);
  const int end = max(0, attn_limit(c, n, min(row0 + 15, a.R - 1) / c.G));
  const int all = (end + 15) / 16, per = (all + pt.splits - 1) / pt.splits;
  const int t0 = pt.split * per, t1 = min(all, t0 + per);
  const char* Kh = c.K.p + pt.b * c.K.b + pt.hk * c.K.h;
  const char* Vh = c.V.p + pt.b * c.V.b + pt.hk * c.V.h;
  float4 qv[W], dv[W];
  f32_quarter<D>(c.Q.p + pt.b * c.Q.b + head * c.Q.h + i * c.Q.n, lane, qv);
  f32_quarter<D>(c.O.p + pt.b * c.O.b + head * c.O.h + i * c.O.n, lane, dv);
  const float* st = a.stat + stat_at((long)pt.b * a.H + head, a.Np, i);
  const float lse = st[0], dsum = st[32];
  f32x4 acc[W];
#pragma unroll
  for (int w = 0; w < W; ++w) acc[w] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int t = t0 + wave; t < t1; t += 4) {
    float4 kv[W], vv[W], kc[4][D / 64];
    const long key = min(t * 16 + lane % 16, n - 1);
    f32_quarter<D>(Kh + key * c.K.n, lane, kv);
    f32_quarter<D>(Vh + key * c.V.n, lane, vv);
    f32_pieces<D>(Kh, c.K.n, t * 16, n - 1, lane, kc);
    const f32x4 sc = f32_rows<D>(kv, qv), dp = f32_rows<D>(vv, dv);
    float ds[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float p = 16 * t + 4 * gr + k < lim ? __builtin_amdgcn_exp2f(fmaf(sc[k], c.scale_log2, -lse)) : 0.f;
      ds[k] = p * (dp[k] - dsum);
    }
    f32_cols<D>(kc, ds, acc);
  }
  float o[W];
  f32_join<D>(os, acc, wave, lane, o);
  const int row = threadIdx.x / 16, rr = row0 + row;
  if (rr >= a.R) return;
  float* out = pt.left >= 0
                   ? a.part + (((long)pt.left * pt.splits + pt.split) * 16 + row) * D
                   : reinterpret_cast<float*>(a.G1.p + pt.b * a.G1.b + (pt.hk * c.G + rr % c.G) * a.G1.h + (rr / c.G) * a.G1.n);
#pragma unroll
  for (int s = 0; s < W / 4; ++s)
    reinterpret_cast<float4*>(out + (threadIdx.x % 16) * W)[s] =
        make_float4(o[4 * s] * c.scale, o[4 * s + 1] * c.scale, o[4 * s + 2] * c.scale, o[4 * s + 3] * c.scale);
}

// ---- dK, dV ----------------------------------------------------------------------------------------------

// The walk of a block of keys: steps of 32 queries, the query heads of its key head one after the other, each from
// the first tile of queries that can see the block.
struct Walk {
  int q0, tiles, t0, t1;  // first query (a multiple of 32), tiles per head, steps of this part
};
__device__ __forceinline__ Walk walk_of(const GradArgs& a, int n, int key0, const Part& pt) {
  const AttnCall& c = a.c;
  Walk w;
  w.q0 = c.causal ? max(0, key0 - (n - c.Nq)) / 32 * 32 : 0;
  w.tiles = key0 < n && w.q0 < c.Nq ? (c.Nq - w.q0 + 31) / 32 : 0;
  const int all = w.tiles * c.G, per = (all + pt.splits - 1) / pt.splits;
  w.t0 = pt.split * per;
  w.t1 = max(w.t0, min(all, w.t0 + per));
  return w;
}

// bf16: a workgroup has 128 keys, in two roles of two waves over the same 64-key columns. Role 0 holds the
// keys' K: S = Q K^T, P, dV^T += dO^T P. Role 1 holds their V: dP = dO V^T, dS = P (dP - D), dK^T += Q^T dS, with
// P from role 0 through LDS one step later, as fp16 (an eighth of the rounding to bf16 that dS takes next). Both
// gradients carry P's factor 2^15 (kLift) to the end. A wave has its SIMD to itself: two 32-key tiles, so that what it reads
// from LDS serves two products (one tile per wave and two waves per SIMD read 1.5 times what the LDS delivers
// while the products run), and the softmax of one tile lies between the products of the other:
//   S_0 | S_1 with P_0 | dV_0 with P_1 and the next step's row operand | dV_1.
constexpr int kDkvBuf = 5;
template <bool CAUSAL>
__global__ __launch_bounds__(256, 1) void attn_dkv_bf16_kernel(const GradArgs a) {
  constexpr int STAGE = 2 * kTile + 1024, DPW = 4, PBUF = 4 * 2048, NBUF = kDkvBuf;
  __shared__ __attribute__((aligned(1024))) char lds[NBUF * STAGE + 2 * PBUF];
  const AttnCall& c = a.c;
  const Part pt = part_of(a.cut, c.Hkv, blockIdx.x);
  const int lane = threadIdx.x % 64, hh = lane / 32;
  const int wave = wave_uniform(threadIdx.x / 64), role = wave / 2, kw = wave % 2;
  const int n = attn_keys(c, pt.b), off = n - c.Nq;
  const int key0 = pt.tile * 128, key = key0 + kw * 64 + lane % 32;  // and key + 32
  const Walk wk = walk_of(a, n, key0, pt);
  const int T = wk.t1 - wk.t0;

  bf16x8 bf[2][8];
  {
    const char* base = role ? c.V.p + pt.b * c.V.b + pt.hk * c.V.h : c.K.p + pt.b * c.K.b + pt.hk * c.K.h;
    const long nstride = role ? c.V.n : c.K.n;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const char* row = base + (long)max(0, min(key + 32 * u, n - 1)) * nstride + 16 * hh;
#pragma unroll
      for (int s = 0; s < 8; ++s) bf[u][s] = *reinterpret_cast<const bf16x8*>(row + 32 * s);
    }
  }
  wait_vm<0>();
  f32x16 acc[2][4];
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int w = 0; w < 4; ++w) acc[u][w] = f32x16{};

  // Loads of a step: waves 0 and 1 the Q rows, waves 2 and 3 the dO rows, 16 rows each.
  const long nstride = role ? c.O.n : c.Q.n, hstride = role ? c.O.h : c.Q.h;
  uint32_t dsrc[DPW];
#pragma unroll
  for (int x = 0; x < DPW; ++x) {
    const int row = 4 * (kw * DPW + x) + lane / 16;
    dsrc[x] = row * (uint32_t)nstride + (((lane % 16) ^ bw_swizzle(row)) << 4);
  }
  const uint32_t lds0 = lds_address(lds);
  const uint32_t dst0 = lds0 + role * kTile + kw * DPW * 1024;
  // The next step to load: its first query, its rows and statistics (pointers that move with it), its stage.
  const int g0 = wk.tiles > 0 ? wk.t0 / wk.tiles : 0, i0 = wk.q0 + (wk.t0 - g0 * wk.tiles) * 32;
  const char* rows = (role ? c.O.p + pt.b * c.O.b : c.Q.p + pt.b * c.Q.b) + ((long)pt.hk * c.G + g0) * hstride +
                     i0 * nstride;
  const char* stats = reinterpret_cast<const char*>(a.stat + (((long)pt.b * a.H + (long)pt.hk * c.G + g0) * a.Np + i0) * 2);
  const long rstep = 32 * nstride, rhead = hstride - (wk.tiles - 1) * rstep;  // to the next tile, the next head's first
  const long shead = 8L * a.Np - (wk.tiles - 1) * 256L;
  int iq = i0, cq = i0, issued = 0;  // cq: the query of the next step to take
  uint32_t dst = dst0, sdst = lds0 + 2 * kTile;
  const uint32_t dst_end = dst0 + NBUF * STAGE;
  uint32_t from[DPW];
  auto aim = [&]() {
#pragma unroll
    for (int x = 0; x < DPW; ++x) from[x] = dsrc[x];
    if (iq + 32 > c.Nq) {  // rows past the last query re-read it (P = 0 there)
#pragma unroll
      for (int x = 0; x < DPW; ++x)
        from[x] -= max(4 * (kw * DPW + x) + lane / 16 - (c.Nq - 1 - iq), 0) * (uint32_t)nstride;
    }
  };
  auto load = [&](int x) { dma16(rows, from[x], dst + x * 1024); };
  auto load_stats = [&]() {  // lse, D of the 32 queries (256 bytes; lanes 16-63 repeat lanes 0-15)
    if (wave == 0) dma16(stats, (lane % 16) * 16, sdst);
  };
  auto loaded = [&]() {  // on to the next step; past the last it is loaded again, to stages that nothing reads
    dst += STAGE, sdst += STAGE;
    if (dst == dst_end) dst -= NBUF * STAGE, sdst -= NBUF * STAGE;
    if (++issued >= T) return;
    iq += 32;
    const bool head_end = iq >= c.Nq;
    rows += head_end ? rhead : rstep;
    stats += head_end ? shead : 256;
    iq = head_end ? wk.q0 : iq;
  };
  auto issue = [&]() {
    aim();
#pragma unroll
    for (int x = 0; x < DPW; ++x) load(x);
    load_stats();
    loaded();
  };

  char* pbase = lds + NBUF * STAGE + kw * 4096 + lane * 16;  // + buffer * PBUF + tile * 2048 + half * 1024
  if (T > 0) {
#pragma unroll
    for (int j = 0; j < NBUF - 2; ++j) issue();
    wait_vm<0>();
    __syncthreads();
  }
  // Iteration t: role 0 takes step t, role 1 step t - 1; the row operand of the step after is read in both. The
  // waves meet before its last products: the loads of step t + NBUF - 1 go where role 1 was in it.
  auto walk = [&](auto role_tag) {
    constexpr int ROLE = decltype(role_tag)::value;
    bf16x8 fa[8];
    auto row_operands = [&](const char* tile) {
#pragma unroll
      for (int s = 0; s < 8; ++s) fa[s] = row_frag(tile, lane % 32, s, hh);
    };
    int buf = 0, back = NBUF - 1;  // stages of steps t and t - 1
    auto meet = [&]() {  // the stage after the next has landed; one more step's loads may be under way
      wait_vm<DPW>();
      __syncthreads();
    };
    auto arrive = [&]() {
      meet();
      issue();
    };
    auto advance = [&]() {
      back = buf;
      buf = buf + 1 == NBUF ? 0 : buf + 1;
    };
    arrive();
    if (ROLE == 1) {
      advance();
      arrive();
    }
    row_operands(lds + ROLE * kTile);
    // (one straight body per role: with a test around it the accumulators move between register files)
    for (int t = ROLE; t < T + ROLE; ++t) {
      const int ahead = buf + 1 == NBUF ? 0 : buf + 1;
      const char* stage = lds + (ROLE ? back : buf) * STAGE;
      char* pb = pbase + ((t - ROLE) & 1) * PBUF;
      const char* tile = stage + (1 - ROLE) * kTile;                          // read transposed
      const char* next = lds + (ROLE ? buf : ahead) * STAGE + ROLE * kTile;  // the next step's rows
      bf16x8 fb[8];
      float lv[16];  // lse less kLift (role 0) or D (role 1) of the step's queries 8 (k / 4) + 4 hh + k % 4
      uint32_t ph[2][8], b2[2][8];  // pairs of fp16 P; of bf16 P or dS
      f32x16 X[2] = {f32x16{}, f32x16{}};
      // P or dS (2^15 of either) of the queries k, k + 1 of tile u. (The empty assembly keeps the work where it stands: the compiler
      // would otherwise sink it past the products it is to lie between.)
      auto middle = [&](int u, int k) {
        if constexpr (ROLE == 0) {
          const float p = __builtin_amdgcn_exp2f(fmaf(X[u][k], c.scale_log2, -lv[k]));
          const float q = __builtin_amdgcn_exp2f(fmaf(X[u][k + 1], c.scale_log2, -lv[k + 1]));
          b2[u][k / 2] = pair_bf16(p, q);
          ph[u][k / 2] = pair_f16(p, q);
          asm volatile("" : "+v"(b2[u][k / 2]), "+v"(ph[u][k / 2]));
          if (k % 8 == 6)
            *reinterpret_cast<uint4*>(pb + u * 2048 + k / 8 * 1024) =
                make_uint4(ph[u][k / 2 - 3], ph[u][k / 2 - 2], ph[u][k / 2 - 1], ph[u][k / 2]);
        } else {
          const f16x2 p = __builtin_bit_cast(f16x2, ph[u][k / 2]);
          b2[u][k / 2] = pair_bf16((float)p[0] * (X[u][k] - lv[k]), (float)p[1] * (X[u][k + 1] - lv[k + 1]));
          asm volatile("" : "+v"(b2[u][k / 2]));
        }
      };
      auto operand = [&](int u, int v) {
        return __builtin_bit_cast(bf16x8, u32x4{b2[u][4 * v], b2[u][4 * v + 1], b2[u][4 * v + 2], b2[u][4 * v + 3]});
      };
      auto hide = [&](int u) {  // P = 0 where the query is before the key
        if (CAUSAL && ROLE == 0 && key0 + kw * 64 + 32 * u + 31 > cq + off) {
          const int late = key + 32 * u - off - cq - 4 * hh;
#pragma unroll
          for (int k = 0; k < 16; ++k) X[u][k] = 8 * (k / 4) + k % 4 >= late ? X[u][k] : -__builtin_inff();
        }
      };
      // (the order between the barriers is the order of issue: a product, then what runs in its shadow)
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        X[0] = mfma_bf16(fa[s], bf[0][s], X[0]);
        fb[s] = tr_frag(tile, s / 2, s % 2, lane);
        if (s < 4) {
          const float4 v = *reinterpret_cast<const float4*>(stage + 2 * kTile + ROLE * 128 + 32 * s + 16 * hh);
          lv[4 * s] = v.x, lv[4 * s + 1] = v.y, lv[4 * s + 2] = v.z, lv[4 * s + 3] = v.w;
        } else if (ROLE == 1) {
          const uint4 v = *reinterpret_cast<const uint4*>(pb + (s / 2 - 2) * 2048 + s % 2 * 1024);
        uint32_t* at = &ph[s / 2 - 2][4 * (s % 2)];
        at[0] = v.x, at[1] = v.y, at[2] = v.z, at[3] = v.w;
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      // (all accumulators at once in their register file: the compiler moved one out and back to make room for S)
      asm volatile("" : "+a"(acc[0][0]), "+a"(acc[0][1]), "+a"(acc[0][2]), "+a"(acc[0][3]), "+a"(acc[1][0]),
                        "+a"(acc[1][1]), "+a"(acc[1][2]), "+a"(acc[1][3]), "+a"(X[0]));
      hide(0);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        X[1] = mfma_bf16(fa[s], bf[1][s], X[1]);
        middle(0, 2 * s);
        __builtin_amdgcn_sched_barrier(0);
      }
      hide(1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        acc[0][s % 4] = mfma_bf16(fb[2 * (s % 4) + s / 4], operand(0, s / 4), acc[0][s % 4]);
        middle(1, 2 * s);
        fa[s] = row_frag(next, lane % 32, s, hh);
        __builtin_amdgcn_sched_barrier(0);
      }
      // the last products, with the next loads between them
      aim();
      meet();
#pragma unroll
      for (int s = 0; s < 8; ++s) {
        acc[1][s % 4] = mfma_bf16(fb[2 * (s % 4) + s / 4], operand(1, s / 4), acc[1][s % 4]);
        if (s < DPW) load(s);
        if (s == DPW) load_stats();
        if (s == DPW + 1) loaded();
        __builtin_amdgcn_sched_barrier(0);
      }
      cq += 32;
      if (cq >= c.Nq) cq = wk.q0;
      advance();
    }
    if (ROLE == 0) arrive();
    wait_vm<0>();  // (loads still under way write to this workgroup's LDS)
  };
  if (T > 0) {
    if (role)
      walk(std::integral_constant<int, 1>{});
    else
      walk(std::integral_constant<int, 0>{});
  }
  __syncthreads();  // every wave is done with the stages
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int k = key + 32 * u;
    if (k >= n) {  // a key that is not there (its column holds the last one's)
#pragma unroll
      for (int w = 0; w < 4; ++w) acc[u][w] = f32x16{};
    }
    const float f = role ? c.scale * kDrop : kDrop;
    if (pt.left >= 0) {
      if (k >= c.Nk) break;
      float* out = a.part + (role ? 0 : a.part2) + (((long)pt.left * pt.splits + pt.split) * 128 + k - key0) * 128;
      store_grad_row<false>(out, acc[u], f, hh, nullptr, nullptr);
    } else {
      const View& g = role ? a.G1 : a.G2;
      rows_from_acc(lds + wave * 8192, acc[u], f, RowBase{g.p + pt.b * g.b + pt.hk * g.h, 0, g.n, 1},
                    key0 + kw * 64 + 32 * u, c.Nk, lane);
    }
  }
}

// fp32: four waves of 16 keys each, query tiles of 32 staged in LDS.
template <int D>
__global__ __launch_bounds__(256, D == 64 ? 1 : 2) void attn_dkv_f32_kernel(const GradArgs a) {
  constexpr int W = D / 16, LD = D + 4, PT = 32 * D / 4 / 256;
  __shared__ __attribute__((aligned(16))) float qs[32 * LD], os[32 * LD];
  __shared__ float st[64];
  const AttnCall& c = a.c;
  const Part pt = part_of(a.cut, c.Hkv, blockIdx.x);
  const int wave = wave_uniform(threadIdx.x / 64), lane = threadIdx.x % 64, gr = lane / 16;
  const int n = attn_keys(c, pt.b), off = n - c.Nq;
  const int key0 = pt.tile * 64, key = key0 + wave * 16 + lane % 16;
  const Walk wk = walk_of(a, n, key0, pt);
  float4 kv[W], vv[W];
  {
    const long k = max(0, min(key, n - 1));
    f32_quarter<D>(c.K.p + pt.b * c.K.b + pt.hk * c.K.h + k * c.K.n, lane, kv);
    f32_quarter<D>(c.V.p + pt.b * c.V.b + pt.hk * c.V.h + k * c.V.n, lane, vv);
  }
  f32x4 dk[W], dv[W];
#pragma unroll
  for (int w = 0; w < W; ++w) dk[w] = dv[w] = f32x4{0.f, 0.f, 0.f, 0.f};
  float4 qn[PT], on[PT];
  float sn = 0.f;
  int g = 0, q = wk.q0;
  if (wk.tiles > 0) {
    g = wk.t0 / wk.tiles;
    q = wk.q0 + wk.t0 % wk.tiles * 32;
  }
  auto fetch = [&]() {
    const int head = pt.hk * c.G + g;
    const char* Qh = c.Q.p + pt.b * c.Q.b + head * c.Q.h;
    const char* Oh = c.O.p + pt.b * c.O.b + head * c.O.h;
#pragma unroll
    for (int x = 0; x < PT; ++x) {
      const int e = threadIdx.x + 256 * x, row = e / (D / 4), at = e % (D / 4);
      const long i = min(q + row, c.Nq - 1);
      qn[x] = reinterpret_cast<const float4*>(Qh + i * c.Q.n)[at];
      on[x] = reinterpret_cast<const float4*>(Oh + i * c.O.n)[at];
    }
    if (threadIdx.x < 64) sn = a.stat[stat_at((long)pt.b * a.H + head, a.Np, q) + threadIdx.x];
  };
  if (wk.t0 < wk.t1) fetch();
  for (int t = wk.t0; t < wk.t1; ++t) {
    __syncthreads();
#pragma unroll
    for (int x = 0; x < PT; ++x) {
      const int e = threadIdx.x + 256 * x, row = e / (D / 4), at = e % (D / 4);
      *reinterpret_cast<float4*>(qs + row * LD + 4 * at) = qn[x];
      *reinterpret_cast<float4*>(os + row * LD + 4 * at) = on[x];
    }
    if (threadIdx.x < 64) st[threadIdx.x] = sn;
    __syncthreads();
    const int q0 = q;
    q += 32;
    if (q >= c.Nq) q = wk.q0, ++g;
    if (t + 1 < wk.t1) fetch();
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const f32x4 sc = f32_rows<D>(qs + 16 * u * LD, kv, lane);
      const f32x4 dp = f32_rows<D>(os + 16 * u * LD, vv, lane);
      float p[4], ds[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {  // query q0 + 16 u + 4 gr + k
        const int row = 16 * u + 4 * gr + k;
        const bool seen = !c.causal || key <= q0 + row + off;
        p[k] = seen ? __builtin_amdgcn_exp2f(fmaf(sc[k], c.scale_log2, -st[row])) : 0.f;
        ds[k] = p[k] * (dp[k] - st[32 + row]);
      }
      f32_cols<D>(os + 16 * u * LD, p, dv, lane);
      f32_cols<D>(qs + 16 * u * LD, ds, dk, lane);
    }
  }
  if (key >= c.Nk) return;
  if (key >= n) {  // a key that is not there (its lane walked with the last one's row)
#pragma unroll
    for (int w = 0; w < W; ++w) dk[w] = dv[w] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  char *pk, *pv;
  if (pt.left >= 0) {
    float* out = a.part + (((long)pt.left * pt.splits + pt.split) * 64 + key - key0) * D;
    pk = reinterpret_cast<char*>(out);
    pv = reinterpret_cast<char*>(out + a.part2);
  } else {
    pk = a.G1.p + pt.b * a.G1.b + pt.hk * a.G1.h + key * a.G1.n;
    pv = a.G2.p + pt.b * a.G2.b + pt.hk * a.G2.h + key * a.G2.n;
  }
  f32_store<D>(pk, dk, c.scale, lane);
  f32_store<D>(pv, dv, 1.f, lane);
}

// fp32, few keys: 16 per workgroup, every fourth sub-tile of 16 queries per wave, straight from memory.
template <int D>
__global__ __launch_bounds__(256, D == 64 ? 1 : 2) void attn_dkv_f32_few_kernel(const GradArgs a) {
  constexpr int W = D / 16;
  __shared__ __attribute__((aligned(16))) float os[4 * 16 * (D + 4)];
  const AttnCall& c = a.c;
  const Part pt = part_of(a.cut, c.Hkv, blockIdx.x);
  const int wave = wave_uniform(threadIdx.x / 64), lane = threadIdx.x % 64, gr = lane / 16;
  const int n = attn_keys(c, pt.b), off = n - c.Nq;
  const int key0 = pt.tile * 16, key = key0 + lane % 16;
  const Walk wk = walk_of(a, n, key0, pt);
  float4 kv[W], vv[W];
  {
    const long k = max(0, min(key, n - 1));
    f32_quarter<D>(c.K.p + pt.b * c.K.b + pt.hk * c.K.h + k * c.K.n, lane, kv);
    f32_quarter<D>(c.V.p + pt.b * c.V.b + pt.hk * c.V.h + k * c.V.n, lane, vv);
  }
  f32x4 dk[W], dv[W];
#pragma unroll
  for (int w = 0; w < W; ++w) dk[w] = dv[w] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int t = 2 * wk.t0 + wave; t < 2 * wk.t1; t += 4) {  // half steps
    const int head = pt.hk * c.G + t / 2 / wk.tiles, q = wk.q0 + t / 2 % wk.tiles * 32 + t % 2 * 16;
    if (q >= c.Nq) continue;
    const char* Qh = c.Q.p + pt.b * c.Q.b + head * c.Q.h;
    const char* Oh = c.O.p + pt.b * c.O.b + head * c.O.h;
    const long i = min(q + lane % 16, c.Nq - 1);
    float4 qv[W], ov[W], qc[4][D / 64], oc[4][D / 64];
    f32_quarter<D>(Qh + i * c.Q.n, lane, qv);
    f32_quarter<D>(Oh + i * c.O.n, lane, ov);
    f32_pieces<D>(Qh, c.Q.n, q, c.Nq - 1, lane, qc);
    f32_pieces<D>(Oh, c.O.n, q, c.Nq - 1, lane, oc);
    const float* st = a.stat + stat_at((long)pt.b * a.H + head, a.Np, q + 4 * gr);
    const float4 l4 = *reinterpret_cast<const float4*>(st), d4 = *reinterpret_cast<const float4*>(st + 32);
    const f32x4 sc = f32_rows<D>(qv, kv), dp = f32_rows<D>(ov, vv);
    const float lse[4] = {l4.x, l4.y, l4.z, l4.w}, dsum[4] = {d4.x, d4.y, d4.z, d4.w};
    float p[4], ds[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {  // query q + 4 gr + k
      const bool seen = !c.causal || key <= q + 4 * gr + k + off;
      p[k] = seen ? __builtin_amdgcn_exp2f(fmaf(sc[k], c.scale_log2, -lse[k])) : 0.f;
      ds[k] = p[k] * (dp[k] - dsum[k]);
    }
    f32_cols<D>(oc, p, dv);
    f32_cols<D>(qc, ds, dk);
  }
  float ok[W], ov[W];
  f32_join<D>(os, dk, wave, lane, ok);
  f32_join<D>(os, dv, wave, lane, ov);
  const int k = key0 + threadIdx.x / 16, c0 = (threadIdx.x % 16) * W;
  if (k >= c.Nk) return;
  if (k >= n) {  // a key that is not there (its lane walked with the last one's row)
#pragma unroll
    for (int w = 0; w < W; ++w) ok[w] = ov[w] = 0.f;
  }
  const float f = c.scale;
  float *pk, *pv;
  if (pt.left >= 0) {
    pk = a.part + (((long)pt.left * pt.splits + pt.split) * 16 + k - key0) * D;
    pv = pk + a.part2;
  } else {
    pk = reinterpret_cast<float*>(a.G1.p + pt.b * a.G1.b + pt.hk * a.G1.h + k * a.G1.n);
    pv = reinterpret_cast<float*>(a.G2.p + pt.b * a.G2.b + pt.hk * a.G2.h + k * a.G2.n);
  }
#pragma unroll
  for (int s = 0; s < W / 4; ++s) {
    reinterpret_cast<float4*>(pk + c0)[s] =
        make_float4(ok[4 * s] * f, ok[4 * s + 1] * f, ok[4 * s + 2] * f, ok[4 * s + 3] * f);
    reinterpret_cast<float4*>(pv + c0)[s] =
        make_float4(ov[4 * s], ov[4 * s + 1], ov[4 * s + 2], ov[4 * s + 3]);
  }
}

// The rows of the cut tiles: sum of their parts, in order. ROWS per tile; a row r is head hk G + r % G, token
// r / G (G = 1: keys). A thread takes four channels. gridDim.y = 2: a second set `part2` further, into out2.
template <typename T, int D, int ROWS>
__global__ __launch_bounds__(256) void attn_sum_kernel(const Cut cut, int Hkv, int G, int rows,
                                                       const float* __restrict__ part, long part2, View out1,
                                                       View out2) {
  const View out = blockIdx.y ? out2 : out1;
  part += blockIdx.y * part2;
  const long e = (long)blockIdx.x * 256 + threadIdx.x;
  const int c = 4 * (int)(e % (D / 4)), row = (int)(e / (D / 4) % ROWS);
  const long left = e / (D / 4) / ROWS;
  int tile;
  long bh;
  cut_tile(cut, cut.whole + (int)left, &tile, &bh);
  const int r = tile * ROWS + row;
  if (r >= rows) return;
  const float* src = part + (left * cut.splits * ROWS + row) * D + c;
  f32x4 s = *reinterpret_cast<const f32x4*>(src);
  for (int k0 = 1; k0 < cut.splits; k0 += 8) {  // eight loads in flight
    f32x4 v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      v[u] = *reinterpret_cast<const f32x4*>(src + (long)min(k0 + u, cut.splits - 1) * ROWS * D);
#pragma unroll
    for (int u = 0; u < 8; ++u) s = k0 + u < cut.splits ? s + v[u] : s;
  }
  const int b = (int)(bh / Hkv), head = (int)(bh % Hkv) * G + r % G;
  T* o = reinterpret_cast<T*>(out.p + b * out.b + head * out.h + (long)(r / G) * out.n) + c;
  #pragma unroll
  for (int k = 0; k < 4; ++k) o[k] = from_f32<T>(s[k]);
}

struct GradPlan {
  int R, Np, rows, keys;  // rows and keys of a tile
  Cut d, q, k;            // the passes of D (bf16), of dQ, of dK and dV
  size_t stat, dsum, dpart, qpart, kpart;  // bytes, 256-aligned; kpart: of dK, and as many of dV
};
size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }
GradPlan grad_plan(const AttnShape& s) {
  GradPlan p{};
  const int G = s.H / s.Hkv, bh = s.B * s.Hkv;
  p.R = s.Nq * G;
  p.Np = (s.Nq + 31) / 32 * 32;
  const int ksteps = (s.Nk + 31) / 32, qsteps = p.Np / 32 * G;
  if (s.bf16) {
    p.rows = p.keys = 128;
  } else {
    const bool little = attn_work(s) < kFewGrad;
    p.rows = little && f32_few((p.R + 63) / 64, bh) ? 16 : 64;
    p.keys = little && f32_few((s.Nk + 63) / 64, bh) ? 16 : 64;
  }
  const int qtiles = (p.R + p.rows - 1) / p.rows, ktiles = (s.Nk + p.keys - 1) / p.keys;
  const double qbytes = p.rows * s.d * 4.0, kbytes = p.keys * s.d * 4.0;
  p.q = s.bf16          ? make_cut(qtiles, bh, s.causal, 2 * kCus, ksteps, 1.6, qbytes, 8)
        : p.rows == 64 ? make_cut(qtiles, bh, s.causal, 2 * kCus, ksteps, 3.0, qbytes, 4)
                       : make_cut(qtiles, bh, s.causal, 2 * kCus, (ksteps + 1) / 2, 2.5, qbytes, 2);
  p.k = s.bf16          ? make_cut(ktiles, bh, s.causal, kCus, qsteps, 1.2, 2 * kbytes, 8)
        : p.keys == 64 ? make_cut(ktiles, bh, s.causal, 2 * kCus, qsteps, 4.0, 2 * kbytes, 4)
                       : make_cut(ktiles, bh, s.causal, 2 * kCus, (qsteps + 1) / 2, 3.5, 2 * kbytes, 2);
  p.stat = up256((size_t)s.B * s.H * p.Np * 2 * sizeof(float));
  if (s.bf16) {
    p.d = make_cut((p.R + 255) / 256, bh, s.causal, 2 * kCus, ksteps, 1.3, 1024, 8);
    p.dsum = up256((size_t)bh * p.R * sizeof(float));
    p.dpart = up256((size_t)cut_left(p.d) * p.d.splits * 256 * sizeof(float));
  }
  p.qpart = up256((size_t)(cut_left(p.q) * p.q.splits * qbytes));
  p.kpart = up256((size_t)(cut_left(p.k) * p.k.splits * kbytes));
  return p;
}

hipError_t launch_sum(const AttnShape& s, const Cut& cut, int per, int G, int rows, int outs, const GradArgs& a,
                      hipStream_t st) {
  const long threads = cut_left(cut) * per * (s.d / 4);  // a multiple of 256: per is one of 16
  const auto k = s.bf16      ? attn_sum_kernel<bf16, 128, 128>
                 : per == 16 ? (s.d == 64 ? attn_sum_kernel<float, 64, 16> : attn_sum_kernel<float, 128, 16>)
                             : (s.d == 64 ? attn_sum_kernel<float, 64, 64> : attn_sum_kernel<float, 128, 64>);
  hipLaunchKernelGGL(k, dim3((unsigned)(threads / 256), outs), dim3(256), 0, st, cut, s.Hkv, G, rows,
                     (const float*)a.part, a.part2, a.G1, a.G2);
  return hipGetLastError();
}

}  // namespace

size_t attn_backward_workspace_bytes(const AttnShape& s) {
  const GradPlan p = grad_plan(s);
  return p.stat + std::max({p.dsum + p.dpart, p.qpart, 2 * p.kpart});
}

hipError_t launch_attn_backward(const AttnShape& s, const HeadView& Q, const HeadView& K, const HeadView& V,
                                const int32_t* kv_len, float scale, const HeadView& O, const float* lse,
                                const HeadView& dO, const HeadView& dQ, const HeadView& dK,
                                const HeadView& dV, void* ws, hipStream_t st) {
  const GradPlan p = grad_plan(s);
  GradArgs a{};
  a.c = attn_call(s, Q, K, V, dO, kv_len, scale);
  a.R = p.R, a.Np = p.Np, a.H = s.H;
  float* stat = (float*)ws;
  a.stat = stat;
  a.lse = lse;
  float* rest = (float*)((char*)ws + p.stat);  // each pass's sums in turn
  const long rows = (long)s.B * s.H * p.Np;
  hipError_t e;
  if (s.bf16) {
    a.cut = p.d;
    a.dsum = rest;
    a.part = (float*)((char*)rest + p.dsum);
    hipLaunchKernelGGL(attn_rowsum_bf16_kernel, dim3(p.d.total), dim3(256), 0, st, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(attn_stat_kernel, dim3((unsigned)((rows + 255) / 256)), dim3(256), 0, st, a, rows, stat);
  } else {
    hipLaunchKernelGGL(attn_rowdot_f32_kernel, dim3((unsigned)std::min<long>((rows + 15) / 16, kRowdotGrid)), dim3(256), 0, st, s.H,
                       s.Nq, p.Np, s.d, rows, view_of(O, false), a.c.O, lse, stat);
  }
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  a.part = rest;
  a.G1 = view_of(dQ, s.bf16);
  a.cut = p.q;
  const auto kq = s.bf16         ? attn_dq_bf16_kernel
                  : p.rows == 16 ? (s.d == 64 ? attn_dq_f32_few_kernel<64> : attn_dq_f32_few_kernel<128>)
                                 : (s.d == 64 ? attn_dq_f32_kernel<64> : attn_dq_f32_kernel<128>);
  hipLaunchKernelGGL(kq, dim3(p.q.total), dim3(256), 0, st, a);
  e = hipGetLastError();
  if (e == hipSuccess && p.qpart) e = launch_sum(s, p.q, p.rows, s.H / s.Hkv, p.R, 1, a, st);
  if (e != hipSuccess) return e;
  a.G1 = view_of(dK, s.bf16), a.G2 = view_of(dV, s.bf16);
  a.cut = p.k;
  a.part2 = (long)(p.kpart / sizeof(float));
  const auto kk = s.bf16         ? (s.causal ? attn_dkv_bf16_kernel<true> : attn_dkv_bf16_kernel<false>)
                  : p.keys == 16 ? (s.d == 64 ? attn_dkv_f32_few_kernel<64> : attn_dkv_f32_few_kernel<128>)
                                 : (s.d == 64 ? attn_dkv_f32_kernel<64> : attn_dkv_f32_kernel<128>);
  hipLaunchKernelGGL(kk, dim3(p.k.total), dim3(256), 0, st, a);
  e = hipGetLastError();
  if (e == hipSuccess && p.kpart) e = launch_sum(s, p.k, p.keys, 1, s.Nk, 2, a, st);
  return e;
}

}  // namespace rola
