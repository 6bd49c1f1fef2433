// Layer norm and RMS norm over the last dimension, with an affine weight and bias that all rows share or
// each group of consecutive rows has of its own (a DiT's modulation per sample), and their gradients.
//   y = xh W + b,  xh = (x - mu) rstd,  rstd = (mean (x - mu)^2 + eps)^(-1/2);  RMS: mu = 0.
//   dB = sum_rows dy,  dW = sum_rows dy xh,
//   g = dy W,  dx = rstd (g - mean g - xh mean(g xh));  RMS: without mean g.
// Bound by HBM: the forward reads x and writes y, the backward reads x and dy and writes dx. So a row is
// read once, into the registers of `TPR` threads (P pieces of eight channels each), and its statistics come
// from there: the mean first, then the squares about it. The waves of a row meet once, with a sum
// and a sum of squares about the wave's own mean each (their squares about the row's mean follow from the two).
// A workgroup walks consecutive rows with its columns of W and b (and the gradient sums) in registers; the
// next row's loads are under way during a row. All sums are fp32. Measured in a kernel trace, bf16: forward
// 75600 x 5120 315 us (4.9 TB/s), 65520 x 1536 73 us and its backward 128 us (4.7 TB/s). The figures at the choices
// below compare two forms at one time; a form that was made faster later takes less than they say.
#include "common.h"
#include "launch.h"
#include "reduce.h"

namespace rola {
namespace {

constexpr int kNormMax = 16384;

// Sum over the wave, in every lane: the four 16-lane rows by permlane swaps, within a row by DPP (no LDS).
template <int CTRL>
__device__ __forceinline__ float dpp_add(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 15, 15, false));
}
__device__ __forceinline__ float wave_sum(float x) {
  x = rows_sum(x);        // lanes l, l^16, l^32, l^48
  x = dpp_add<0xB1>(x);   // l ^ 1
  x = dpp_add<0x4E>(x);   // l ^ 2
  x = dpp_add<0x141>(x);  // mirror of 8 lanes
  return dpp_add<0x140>(x);  // mirror of 16
}

// Eight consecutive elements as loaded.
template <typename T>
struct Raw8 {
  uint4 u[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ void raw_load(const T* p, Raw8<T>& r) {
#pragma unroll
  for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.u[i] = reinterpret_cast<const uint4*>(p)[i];
}
template <typename T>
__device__ __forceinline__ void unpack(const Raw8<T>& r, float v[8]) {
  load8(reinterpret_cast<const T*>(&r), v);
}

// Columns of W or b (fp32 or bf16), `fill` where there is none.
__device__ __forceinline__ void load_param(const void* p, bool half, long at, float fill, float v[8]) {
  if (!p) {
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = fill;
  } else if (half) {
    load8((const bf16*)p + at, v);
  } else {
    load8((const float*)p + at, v);
  }
}

struct NormArgs {
  long per;       // rows per group
  long chunk;     // rows per workgroup
  int d;
  int rms, whalf;
  long ldx, ldy, ldo;  // row strides of x, dy and the output
  float eps;
  const void* x;
  const void* w;
  const void* b;
  const void* dy;
  void* out;      // y or dx
  float* mean;
  float* rstd;
  float* part;    // [groups][chunks][2 d]: sums of dW, dB
};

// Threads of a workgroup: one row of TPR threads, or four rows of a wave each side by side.
template <int TPR>
constexpr int norm_threads() { return TPR < 256 ? 256 : TPR; }

template <typename T, int TPR, int P>
__global__ __launch_bounds__(norm_threads<TPR>()) void norm_fwd_kernel(const NormArgs a) {
  constexpr int THREADS = norm_threads<TPR>(), RPB = THREADS / TPR, WPR = TPR / 64;
  __shared__ float2 meet[2][WPR];
  const int slot = wave_uniform(threadIdx.x / TPR), tid = threadIdx.x % TPR, d = a.d;
  const int wr = wave_uniform(tid / 64);
  const long r0 = blockIdx.x * a.chunk, r1 = min(a.per, r0 + a.chunk);
  const long base = blockIdx.y * a.per;  // first row of the group
  int col[P];
  float w[P][8], b[P][8];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    col[p] = 8 * (tid + p * TPR);
    if (col[p] < d) {
      load_param(a.w, a.whalf, (long)blockIdx.y * d + col[p], 1.f, w[p]);
      load_param(a.b, a.whalf, (long)blockIdx.y * d + col[p], 0.f, b[p]);
    }
  }
  const T* X = (const T*)a.x + base * a.ldx;
  T* Y = (T*)a.out + base * a.ldo;
  const float inv = 1.f / d;
  Raw8<T> nxt[P];
  auto fetch = [&](long r) {
    const T* row = X + min(r, r1 - 1) * a.ldx;
#pragma unroll
    for (int p = 0; p < P; ++p)
      if (col[p] < d) raw_load(row + col[p], nxt[p]);
  };
  fetch(r0 + slot);
  // (every wave of the workgroup takes the same number of turns: rows past the chunk repeat its last)
  int turn = 0;
  for (long rr = r0; rr < r1; rr += RPB, turn ^= 1) {
    const long r = rr + slot;
    float v[P][8];
#pragma unroll
    for (int p = 0; p < P; ++p)
      if (col[p] < d) unpack(nxt[p], v[p]);
    fetch(r + RPB);
    float mu = 0.f, m2 = 0.f;
    if (!a.rms) {
      float s = 0.f;
#pragma unroll
      for (int p = 0; p < P; ++p)
        if (col[p] < d)
#pragma unroll
          for (int k = 0; k < 8; ++k) s += v[p][k];
      s = wave_sum(s);
      // channels of this wave (whole pieces of eight)
      int cnt = 0;
#pragma unroll
      for (int p = 0; p < P; ++p) cnt += min(max(d - 8 * (64 * wr + p * TPR), 0), 512);
      const float mw = s / max(cnt, 1);
#pragma unroll
      for (int p = 0; p < P; ++p)
        if (col[p] < d)
#pragma unroll
          for (int k = 0; k < 8; ++k) m2 = fmaf(v[p][k] - mw, v[p][k] - mw, m2);
      m2 = wave_sum(m2);
      mu = mw;
      if constexpr (WPR > 1) {
        if (threadIdx.x % 64 == 0) meet[turn][wr] = make_float2(s, m2);
        __syncthreads();
        float2 o[WPR];
        s = 0.f;
#pragma unroll
        for (int i = 0; i < WPR; ++i) {
          o[i] = meet[turn][i];
          s += o[i].x;
        }
        mu = s / d;  // (a rounded 1 / d would leave (2^-25 mu)^2 in the squares of a constant row)
        m2 = 0.f;
#pragma unroll
        for (int i = 0; i < WPR; ++i) {
          int n = 0;
#pragma unroll
          for (int p = 0; p < P; ++p) n += min(max(d - 8 * (64 * i + p * TPR), 0), 512);
          const float e = o[i].x / max(n, 1) - mu;
          m2 += fmaf(n * e, e, o[i].y);
        }
      }
    } else {
#pragma unroll
      for (int p = 0; p < P; ++p)
        if (col[p] < d)
#pragma unroll
          for (int k = 0; k < 8; ++k) m2 = fmaf(v[p][k], v[p][k], m2);
      m2 = wave_sum(m2);
      if constexpr (WPR > 1) {
        if (threadIdx.x % 64 == 0) meet[turn][wr] = make_float2(m2, 0.f);
        __syncthreads();
        m2 = 0.f;
#pragma unroll
        for (int i = 0; i < WPR; ++i) m2 += meet[turn][i].x;
      }
    }
    const float rs = 1.f / sqrtf(m2 * inv + a.eps);
    if (r < r1) {
      T* row = Y + r * a.ldo;
#pragma unroll
      for (int p = 0; p < P; ++p)
        if (col[p] < d) {
          float o[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) o[k] = fmaf((v[p][k] - mu) * rs, w[p][k], b[p][k]);
          store8(row + col[p], o);
        }
      if (tid == 0) {
        if (a.mean) a.mean[base + r] = mu;
        if (a.rstd) a.rstd[base + r] = rs;
      }
    }
  }
}

// The backward of a chunk of rows: dx, and the chunk's sums of dy xh and dy into its partial. (The registers are left to
// the compiler: with a third wave per SIMD forced where it takes two, rows spill, and bf16 65536 x 1536 takes 140 us
// instead of 139, 8192 x 12288 158 instead of 147.)
template <typename T, int TPR, int P>
__global__ __launch_bounds__(norm_threads<TPR>()) void norm_bwd_kernel(const NormArgs a) {
  constexpr int THREADS = norm_threads<TPR>(), RPB = THREADS / TPR, WPR = TPR / 64;
  __shared__ float2 meet[2][WPR];
  __shared__ float sums[RPB > 1 ? THREADS : 1][8];
  const int slot = wave_uniform(threadIdx.x / TPR), tid = threadIdx.x % TPR, d = a.d;
  const int wr = wave_uniform(tid / 64);
  const long r0 = blockIdx.x * a.chunk, r1 = min(a.per, r0 + a.chunk);
  const long base = blockIdx.y * a.per;
  int col[P];
  float w[P][8], sw[P][8], sb[P][8];
#pragma unroll
  for (int p = 0; p < P; ++p) {
    col[p] = 8 * (tid + p * TPR);
    if (col[p] < d) load_param(a.w, a.whalf, (long)blockIdx.y * d + col[p], 1.f, w[p]);
#pragma unroll
    for (int k = 0; k < 8; ++k) sw[p][k] = sb[p][k] = 0.f;
  }
  const T* X = (const T*)a.x + base * a.ldx;
  const T* DY = (const T*)a.dy + base * a.ldy;
  T* DX = (T*)a.out + base * a.ldo;
  const float inv = 1.f / d;
  Raw8<T> nx[P], ny[P];
  float nmu = 0.f, nrs = 0.f;
  auto fetch = [&](long r) {
    r = min(r, r1 - 1);
#pragma unroll
    for (int p = 0; p < P; ++p)
      if (col[p] < d) {
        raw_load(X + r * a.ldx + col[p], nx[p]);
        raw_load(DY + r * a.ldy + col[p], ny[p]);
      }
    if (!a.rms) nmu = a.mean[base + r];
    nrs = a.rstd[base + r];
  };
  fetch(r0 + slot);
  int turn = 0;
  for (long rr = r0; rr < r1; rr += RPB, turn ^= 1) {
    const long r = rr + slot;
    Raw8<T> cx[P], cy[P];  // the row as loaded, taken apart twice: in bf16 half the registers of its values
    float c1 = 0.f, c2 = 0.f;
    const float mu = nmu, rs = nrs;
#pragma unroll
    for (int p = 0; p < P; ++p)
      if (col[p] < d) cx[p] = nx[p], cy[p] = ny[p];
    fetch(r + RPB);
#pragma unroll
    for (int p = 0; p < P; ++p)
      if (col[p] < d) {
        float xh[8], g[8];
        unpack(cx[p], xh);
        unpack(cy[p], g);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          xh[k] = (xh[k] - mu) * rs;
          if (RPB == 1 || r < r1) {
            sw[p][k] = fmaf(g[k], xh[k], sw[p][k]);
            sb[p][k] += g[k];
          }
          g[k] *= w[p][k];
          c1 += g[k];
          c2 = fmaf(g[k], xh[k], c2);
        }
      }
    c1 = wave_sum(c1);
    c2 = wave_sum(c2);
    if constexpr (WPR > 1) {
      if (threadIdx.x % 64 == 0) meet[turn][wr] = make_float2(c1, c2);
      __syncthreads();
      c1 = c2 = 0.f;
#pragma unroll
      for (int i = 0; i < WPR; ++i) {
        const float2 o = meet[turn][i];
        c1 += o.x;
        c2 += o.y;
      }
    }
    c1 = a.rms ? 0.f : c1 * inv;
    c2 *= inv;
    if (r < r1) {
#pragma unroll
      for (int p = 0; p < P; ++p)
        if (col[p] < d) {
          float x[8], g[8], o[8];
          unpack(cx[p], x);
          unpack(cy[p], g);
#pragma unroll
          for (int k = 0; k < 8; ++k) o[k] = rs * (fmaf(g[k], w[p][k], -c1) - (x[k] - mu) * rs * c2);
          store8(DX + r * a.ldo + col[p], o);
        }
    }
  }
  float* part = a.part + ((long)blockIdx.y * gridDim.x + blockIdx.x) * 2 * d;
#pragma unroll
  for (int p = 0; p < P; ++p)
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      float s[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) s[k] = which ? sb[p][k] : sw[p][k];
      if constexpr (RPB > 1) {  // the rows side by side, in order
        __syncthreads();
        store8(sums[threadIdx.x], s);
        __syncthreads();
        if (slot) continue;
#pragma unroll
        for (int i = 1; i < RPB; ++i)
#pragma unroll
          for (int k = 0; k < 8; ++k) s[k] += sums[i * TPR + tid][k];
      }
      if (col[p] < d) store8(part + which * d + col[p], s);
    }
}

// Threads per row. Up to 2048 channels a wave, which has no meeting with others per row (forward, 65520 rows of
// 1536: 85 us, 100 with 256 threads; backward 147 and 156); for few rows 256, whose chain of loads and sums is a
// quarter as long. Beyond, 256 or 512: forward 75600 x 5120 314 us with 256, 390 with 512, backward 499
// and 487; 8192 x 8192 backward 103 and 100. Rows of fewer than 512 channels leave lanes of their wave idle: 96 x 2^20
// bf16 values as rows of 512, 256, 128, 64 channels take 82, 96, 176, 336 us forward and 136, 195, 327, 562 backward.
int norm_row_threads(long rows, int d, bool bwd) {
  if (d > 8192) return 512;
  if (d > 2048) return bwd ? 512 : 256;
  return rows < kCus ? 256 : 64;
}

// Pieces per thread that rows of d channels come to with the threads that norm_row_threads gives them: what there are
// kernels for. 256 threads take up to 2048 channels (few rows) in either direction and the forward's up to 8192, 512
// the backward's from there on and the forward's beyond 8192.
template <bool BWD, int TPR>
constexpr int kLeastPieces = TPR == 512 && !BWD ? 3 : 1;
template <bool BWD, int TPR>
constexpr int kMostPieces = TPR == 256 && BWD ? 1 : 4;

template <typename T, bool BWD, int TPR, int P = kLeastPieces<BWD, TPR>>
hipError_t launch_norm_p(const NormArgs& a, dim3 grid, hipStream_t st) {
  if ((a.d / 8 + TPR - 1) / TPR == P) {
    if constexpr (BWD)
      hipLaunchKernelGGL((norm_bwd_kernel<T, TPR, P>), grid, dim3(norm_threads<TPR>()), 0, st, a);
    else
      hipLaunchKernelGGL((norm_fwd_kernel<T, TPR, P>), grid, dim3(norm_threads<TPR>()), 0, st, a);
    return hipGetLastError();
  }
  if constexpr (P < kMostPieces<BWD, TPR>) return launch_norm_p<T, BWD, TPR, P + 1>(a, grid, st);
  return hipErrorInvalidConfiguration;
}

template <bool BWD>
hipError_t launch_norm_t(bool bf, const NormArgs& a, int tpr, dim3 grid, hipStream_t st) {
  if (bf)
    return tpr == 64    ? launch_norm_p<bf16, BWD, 64>(a, grid, st)
           : tpr == 256 ? launch_norm_p<bf16, BWD, 256>(a, grid, st)
                        : launch_norm_p<bf16, BWD, 512>(a, grid, st);
  return tpr == 64    ? launch_norm_p<float, BWD, 64>(a, grid, st)
         : tpr == 256 ? launch_norm_p<float, BWD, 256>(a, grid, st)
                      : launch_norm_p<float, BWD, 512>(a, grid, st);
}

// Workgroups per group of rows, each of at least one turn of rows. The forward takes many short ones (16 per CU of
// 256 threads a row: 4096 channels 108 us, with 8 115; 512 threads: 16384 channels 56 with 4, 67 with 16), the
// backward two per CU, as each leaves a partial of 2 d sums (65520 x 1536: 147 us, with 4 155, with 16 207).
struct NormPlan {
  int tpr;
  long chunk;
  int chunks;
};
NormPlan norm_plan(const NormShape& s, bool bwd) {
  const long per = s.rows / s.groups;
  const int tpr = norm_row_threads(s.rows, s.d, bwd), side = tpr < 256 ? 256 / tpr : 1;
  const long want = (bwd ? 2 : tpr == 64 ? 8 : tpr == 256 ? 16 : 4) * kCus;
  const long n = (want + s.groups - 1) / s.groups;
  const long chunk = ((per + n - 1) / n + side - 1) / side * side;
  return {tpr, chunk, (int)((per + chunk - 1) / chunk)};
}

}  // namespace

int norm_max_channels() { return kNormMax; }

hipError_t launch_norm(const NormShape& s, const void* X, long ldx, const void* W, const void* Bias,
                       float eps, void* Y, long ldy, float* mean, float* rstd, hipStream_t st) {
  const NormPlan pl = norm_plan(s, false);
  NormArgs a{};
  a.per = s.rows / s.groups, a.chunk = pl.chunk, a.d = s.d, a.rms = s.rms, a.whalf = s.wbf16;
  a.ldx = ldx, a.ldo = ldy, a.eps = eps;
  a.x = X, a.w = W, a.b = Bias, a.out = Y, a.mean = mean, a.rstd = rstd;
  return launch_norm_t<false>(s.bf16, a, pl.tpr, dim3(pl.chunks, s.groups), st);
}

size_t norm_backward_workspace_bytes(const NormShape& s) {
  return (size_t)norm_plan(s, true).chunks * s.groups * 2 * s.d * sizeof(float);
}

hipError_t launch_norm_backward(const NormShape& s, const void* X, long ldx, const void* W,
                                const float* mean, const float* rstd, const void* dY, long ldy, void* dX,
                                long lddx, float* dW, float* dB, void* ws, hipStream_t st) {
  const NormPlan pl = norm_plan(s, true);
  NormArgs a{};
  a.per = s.rows / s.groups, a.chunk = pl.chunk, a.d = s.d, a.rms = s.rms, a.whalf = s.wbf16;
  a.ldx = ldx, a.ldy = ldy, a.ldo = lddx;
  a.x = X, a.w = W, a.dy = dY, a.out = dX, a.mean = const_cast<float*>(mean), a.rstd = const_cast<float*>(rstd);
  a.part = (float*)ws;
  const hipError_t e = launch_norm_t<true>(s.bf16, a, pl.tpr, dim3(pl.chunks, s.groups), st);
  if (e != hipSuccess || !dW) return e;
  return launch_chunk_reduce(2 * s.d, s.d, 2L * s.d, 1, s.groups, pl.chunks, (const float*)ws, dW, dB, st);
}

}  // namespace rola
