// Layer norm over the columns of every row, and its gradients.
//
//   m = mean(x), r = 1 / sqrt(mean((x - m)^2) + eps), y = (x - m) r gamma + beta
//   g = dy gamma, xh = (x - m) r:  dx = r (g - mean(g) - xh mean(g xh)) [+ add],
//   dgamma = sum over rows of dy xh, dbeta = sum over rows of dy
//
// Memory bounds both passes: a row is read once into registers (the variance from the differences to the mean, not from
// sums of squares, which cancel), reduced by the lanes that hold it, and written once.  LPR lanes share a row, each with NV
// 16-byte vectors of it; a row of more than 256 vectors takes a workgroup of four waves.  The weights' gradients are summed in
// registers over a workgroup's rows, at most kMostSums rows to a sum, joined in LDS and written as one partial row for each
// workgroup; a second kernel adds those in double.  No atomics: the same inputs give the same bits.
// Measured: 3.2 M rows of 128 bf16 forward 347 us, 4.7 TB/s; 500 000 rows of 256 fp32 backward with `add` 380 us, 5.4 TB/s, the join 7 us;
// 1000 rows of 172 fp32 5.5 us, two dependent reductions behind one load.
#include <algorithm>

#include "dgc_join.h"
#include "dgc_ops.h"

namespace dgc {
namespace {

using ops::Elem;

constexpr int kMaxF = 8192;
constexpr int kBlocks = 2048;       // workgroups of a forward pass at most: 8 a CU
constexpr int kSumBlocks = 1024;    // workgroups of a backward pass, and so partial rows, unless kMostSums asks for more
constexpr int kMostSums = 512;      // rows that one fp32 register adds up: its error grows with their root, 5e-7 at 512

struct NormArgs {
  const void* x; int64_t ldx;
  const void* dy; int64_t lddy;
  const void* add; int64_t ldadd;
  void* out; int64_t ldo;         // y, or dx
  const float* gamma;
  const float* beta;
  float* mean;
  float* rstd;
  float* partial;                 // [workgroups][2][F], or nullptr: no gradients of the weights
  int64_t R;
  int32_t F;
  float eps;
};

// Sums over the lanes of a row, the same on each of them.  Rows of a whole workgroup (LPR = 256) go through LDS: `slot`
// alternates, so that one barrier a sum is enough.
template <int LPR, int K>
__device__ __forceinline__ void row_sums(float (&s)[K], float* lds, int& slot) {
#pragma unroll
  for (int k = 0; k < K; ++k) {
#pragma unroll
    for (int m = (LPR < 64 ? LPR : 64) / 2; m >= 1; m >>= 1) s[k] += __shfl_xor(s[k], m);
  }
  if constexpr (LPR == 256) {
    float* w = lds + slot * 8;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int k = 0; k < K; ++k) w[(threadIdx.x >> 6) * 2 + k] = s[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) s[k] = (w[k] + w[2 + k]) + (w[4 + k] + w[6 + k]);
    slot ^= 1;
  }
}

template <int LPR, int NV, int VN>
__device__ __forceinline__ void load_weights(const float* w, int sub, int F, float none, float (&out)[NV][VN]) {
#pragma unroll
  for (int j = 0; j < NV; ++j) {
#pragma unroll
    for (int i = 0; i < VN; ++i) {
      const int col = (sub + j * LPR) * VN + i;
      out[j][i] = w && col < F ? w[col] : none;
    }
  }
}

// U rows in flight for every group of LPR lanes.
template <class T, int LPR, int NV, int U>
__global__ __launch_bounds__(256) void k_norm_forward(NormArgs a) {
  constexpr int VN = Elem<T>::kPer, GROUPS = 256 / LPR;
  __shared__ float lds[16];
  int slot = 0;
  const int sub = threadIdx.x % LPR, grp = threadIdx.x / LPR, F = a.F;
  float gamma[NV][VN], beta[NV][VN];
  load_weights<LPR, NV, VN>(a.gamma, sub, F, 1.f, gamma);
  load_weights<LPR, NV, VN>(a.beta, sub, F, 0.f, beta);
  const float n = (float)F;
  for (int64_t base = (int64_t)blockIdx.x * (GROUPS * U); base < a.R; base += (int64_t)gridDim.x * (GROUPS * U)) {
    float x[U][NV][VN];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t r = base + u * GROUPS + grp;
      const T* row = static_cast<const T*>(a.x) + r * a.ldx;
#pragma unroll
      for (int j = 0; j < NV; ++j) ops::load_vec(row, (sub + j * LPR) * VN, r < a.R ? F : 0, x[u][j]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t r = base + u * GROUPS + grp;
      float s[1] = {0.f};
#pragma unroll
      for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int i = 0; i < VN; ++i) s[0] += x[u][j][i];
      }
      row_sums<LPR>(s, lds, slot);
      const float m = s[0] / n;
      s[0] = 0.f;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int i = 0; i < VN; ++i) {
          const float d = (sub + j * LPR) * VN + i < F ? x[u][j][i] - m : 0.f;
          x[u][j][i] = d;
          s[0] = fmaf(d, d, s[0]);
        }
      }
      row_sums<LPR>(s, lds, slot);
      const float rstd = 1.f / sqrtf(s[0] / n + a.eps);
      if (r < a.R) {
        T* out = static_cast<T*>(a.out) + r * a.ldo;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
#pragma unroll
          for (int i = 0; i < VN; ++i) x[u][j][i] = fmaf(x[u][j][i] * rstd, gamma[j][i], beta[j][i]);
          ops::store_vec(out, (sub + j * LPR) * VN, F, x[u][j]);
        }
        if (sub == 0 && a.mean) a.mean[r] = m;
        if (sub == 0 && a.rstd) a.rstd[r] = rstd;
      }
    }
  }
}

template <class T, int LPR, int NV, int U>
__global__ __launch_bounds__(256) void k_norm_backward(NormArgs a) {
  constexpr int VN = Elem<T>::kPer, GROUPS = 256 / LPR;
  __shared__ float lds[16];
  __shared__ float joined[GROUPS > 1 ? 256 * NV * VN : 1];
  int slot = 0;
  const int sub = threadIdx.x % LPR, grp = threadIdx.x / LPR, F = a.F;
  float gamma[NV][VN], dgamma[NV][VN], dbeta[NV][VN];
  load_weights<LPR, NV, VN>(a.gamma, sub, F, 1.f, gamma);
#pragma unroll
  for (int j = 0; j < NV; ++j) {
#pragma unroll
    for (int i = 0; i < VN; ++i) dgamma[j][i] = dbeta[j][i] = 0.f;
  }
  const float n = (float)F;
  for (int64_t base = (int64_t)blockIdx.x * (GROUPS * U); base < a.R; base += (int64_t)gridDim.x * (GROUPS * U)) {
    float x[U][NV][VN], dy[U][NV][VN], m[U], rstd[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t r = base + u * GROUPS + grp;
      const T* row = static_cast<const T*>(a.x) + r * a.ldx;
      const T* drow = static_cast<const T*>(a.dy) + r * a.lddy;
      m[u] = r < a.R ? a.mean[r] : 0.f;
      rstd[u] = r < a.R ? a.rstd[r] : 0.f;
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        ops::load_vec(row, (sub + j * LPR) * VN, r < a.R ? F : 0, x[u][j]);
        ops::load_vec(drow, (sub + j * LPR) * VN, r < a.R ? F : 0, dy[u][j]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t r = base + u * GROUPS + grp;
      float s[2] = {0.f, 0.f};
#pragma unroll
      for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int i = 0; i < VN; ++i) {
          const float xh = (sub + j * LPR) * VN + i < F ? (x[u][j][i] - m[u]) * rstd[u] : 0.f;
          const float g = dy[u][j][i] * gamma[j][i];
          x[u][j][i] = xh;
          s[0] += g;
          s[1] = fmaf(g, xh, s[1]);
          dgamma[j][i] = fmaf(dy[u][j][i], xh, dgamma[j][i]);
          dbeta[j][i] += dy[u][j][i];
        }
      }
      row_sums<LPR>(s, lds, slot);
      const float mg = s[0] / n, mgx = s[1] / n;
      if (r < a.R) {
        T* out = static_cast<T*>(a.out) + r * a.ldo;
        const T* add = static_cast<const T*>(a.add) + r * a.ldadd;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const int col = (sub + j * LPR) * VN;
          float more[VN] = {};
          if (a.add) ops::load_vec(add, col, F, more);
#pragma unroll
          for (int i = 0; i < VN; ++i) {
            const float d = dy[u][j][i] * gamma[j][i] - mg;
            x[u][j][i] = fmaf(rstd[u], fmaf(-x[u][j][i], mgx, d), more[i]);
          }
          ops::store_vec(out, col, F, x[u][j]);
        }
      }
    }
  }
  if (!a.partial) return;
  // the sums of the workgroup's groups, in their order
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float* to = a.partial + ((int64_t)blockIdx.x * 2 + which) * F;
    if constexpr (GROUPS == 1) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int i = 0; i < VN; ++i) {
          const int col = (sub + j * LPR) * VN + i;
          if (col < F) to[col] = which ? dbeta[j][i] : dgamma[j][i];
        }
      }
    } else {
      constexpr int W = LPR * NV * VN;   // columns that a group holds
      __syncthreads();
#pragma unroll
      for (int j = 0; j < NV; ++j) {
#pragma unroll
        for (int i = 0; i < VN; ++i) joined[grp * W + (sub + j * LPR) * VN + i] = which ? dbeta[j][i] : dgamma[j][i];
      }
      __syncthreads();
      for (int col = threadIdx.x; col < F; col += 256) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < GROUPS; ++k) s += joined[k * W + col];
        to[col] = s;
      }
    }
  }
}

struct Shape { int lpr, nv, u; };   // lanes a row, vectors a lane, rows in flight

// As few lanes a row as hold it in one vector each, up to a wave; then up to four vectors a lane; then a workgroup a row.
Shape shape_of(int32_t F, int per) {
  const int vecs = (F + per - 1) / per;
  int lpr = 4;
  while (lpr < vecs && lpr < 64) lpr *= 2;
  if (vecs <= 64) return {lpr, 1, 4};
  if (vecs <= 128) return {64, 2, 2};
  if (vecs <= 192) return {64, 3, 1};
  if (vecs <= 256) return {64, 4, 1};
  if (vecs <= 512) return {256, 2, 1};
  if (vecs <= 768) return {256, 3, 1};
  if (vecs <= 1024) return {256, 4, 1};
  return {256, 8, 1};
}

// Workgroups of a backward pass, for either element type: the workspace depends on it, so it counts with the wider rows.
int64_t sum_blocks(int64_t R, int32_t F, int per) {
  const Shape s = shape_of(F, per);
  const int64_t rows = (int64_t)(256 / s.lpr) * s.u, turns = (R + rows - 1) / rows;
  // Of wide rows, fewer: their partial rows are traffic (868 rows of 6417 fp32: 78 us with as many as 1024, 41 with 256), but two vectors a
  // lane leave registers for more waves (30 000 rows of 4096 bf16: 241 us with 512, 393 with 256).
  const int64_t fill = s.lpr < 256 ? kSumBlocks : s.nv == 2 ? kSumBlocks / 2 : kSumBlocks / 4;
  return std::max(std::min<int64_t>(turns, fill), (turns * s.u + kMostSums - 1) / kMostSums);
}

template <class T, bool BACK>
void launch(const NormArgs& a, int64_t blocks, hipStream_t st) {
  const Shape s = shape_of(a.F, Elem<T>::kPer);
  auto go = [&](auto fwd, auto bwd) {
    if (BACK) hipLaunchKernelGGL(bwd, (unsigned)blocks, 256, 0, st, a);
    else hipLaunchKernelGGL(fwd, (unsigned)blocks, 256, 0, st, a);
  };
#define DGC_NORM(L, N, U) \
  if (s.lpr == L && s.nv == N) return go(k_norm_forward<T, L, N, U>, k_norm_backward<T, L, N, U>)
  DGC_NORM(4, 1, 4);
  DGC_NORM(8, 1, 4);
  DGC_NORM(16, 1, 4);
  DGC_NORM(32, 1, 4);
  DGC_NORM(64, 1, 4);
  DGC_NORM(64, 2, 2);
  DGC_NORM(64, 3, 1);
  DGC_NORM(64, 4, 1);
  DGC_NORM(256, 2, 1);
  DGC_NORM(256, 3, 1);
  DGC_NORM(256, 4, 1);
  if constexpr (Elem<T>::kPer == 4) DGC_NORM(256, 8, 1);
#undef DGC_NORM
}

const char* check(int64_t R, int32_t F, int32_t dtype, float eps) {
  if (dtype != DGC_DTYPE_F32 && dtype != DGC_DTYPE_BF16) return "norm: unknown dtype";
  if (R < 0 || F < 1 || F > kMaxF) return "norm: R must be >= 0 and F in [1, 8192]";
  if (!(eps >= 0.f)) return "norm: eps must be >= 0";
  return nullptr;
}

}  // namespace
}  // namespace dgc

using namespace dgc;

extern "C" {

int64_t dgc_norm_workspace_bytes(int64_t R, int32_t F) {
  if (R < 0 || F < 1 || F > kMaxF) return -1;
  return 8 * (int64_t)F * std::max<int64_t>(1, std::max(sum_blocks(R, F, 4), sum_blocks(R, F, 8)));
}

dgc_status_t dgc_norm_forward(const void* x, int64_t ldx, int64_t R, int32_t F, int32_t dtype, const float* gamma,
                              const float* beta, float eps, void* y, int64_t ldy, float* mean, float* rstd, void* stream) {
  if (const char* msg = check(R, F, dtype, eps)) return ops::refuse(DGC_ERR_INVALID_ARG, msg);
  const int e = ops::elem_bytes(dtype);
  if (!ops::good_rows(x, R, F, ldx, e) || !ops::good_rows(y, R, F, ldy, e))
    return ops::refuse(DGC_ERR_INVALID_ARG, "norm: x, y need a 16-byte aligned base and a pitch >= F that is a multiple of 16 bytes");
  if (!ops::same_place(x, ldx, y, ldy) && ops::share(x, ldx, e, F, y, ldy, e, F, R))
    return ops::refuse(DGC_ERR_INVALID_ARG, "norm: y is x itself or apart from it");
  if (R == 0) return DGC_OK;
  NormArgs a{};
  a.x = x; a.ldx = ldx; a.out = y; a.ldo = ldy; a.gamma = gamma; a.beta = beta; a.mean = mean; a.rstd = rstd;
  a.R = R; a.F = F; a.eps = eps;
  const Shape s = shape_of(F, 16 / e);
  const int64_t rows = (int64_t)(256 / s.lpr) * s.u, blocks = std::min<int64_t>((R + rows - 1) / rows, kBlocks);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == DGC_DTYPE_F32) launch<float, false>(a, blocks, st);
  else launch<uint16_t, false>(a, blocks, st);
  return ops::launched("norm");
}

dgc_status_t dgc_norm_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, const float* mean, const float* rstd,
                               int64_t R, int32_t F, int32_t dtype, const float* gamma, const void* add, int64_t ldadd, void* dx,
                               int64_t lddx, float* dgamma, float* dbeta, void* workspace, int64_t workspace_bytes, void* stream) {
  if (const char* msg = check(R, F, dtype, 0.f)) return ops::refuse(DGC_ERR_INVALID_ARG, msg);
  const int e = ops::elem_bytes(dtype);
  if (!ops::good_rows(dy, R, F, lddy, e) || !ops::good_rows(x, R, F, ldx, e) || !ops::good_rows(dx, R, F, lddx, e) ||
      (add && !ops::good_rows(add, R, F, ldadd, e)))
    return ops::refuse(DGC_ERR_INVALID_ARG, "norm: dy, x, add, dx need a 16-byte aligned base and a pitch >= F that is a multiple of 16 bytes");
  if (R > 0 && (!mean || !rstd)) return ops::refuse(DGC_ERR_INVALID_ARG, "norm: the backward pass needs the forward's mean and rstd");
  const struct { const void* p; int64_t ld; } in[3] = {{dy, lddy}, {x, ldx}, {add, ldadd}};
  for (const auto& t : in) {
    if (!ops::same_place(t.p, t.ld, dx, lddx) && ops::share(t.p, t.ld, e, F, dx, lddx, e, F, R))
      return ops::refuse(DGC_ERR_INVALID_ARG, "norm: dx is one of its inputs itself or apart from them");
  }
  const bool sums = dgamma || dbeta;
  if (sums && (!workspace || !ops::aligned16(workspace) || workspace_bytes < dgc_norm_workspace_bytes(R, F)))
    return ops::refuse(DGC_ERR_INVALID_ARG, "norm: workspace missing, too small (dgc_norm_workspace_bytes) or not 16-byte aligned");
  NormArgs a{};
  a.x = x; a.ldx = ldx; a.dy = dy; a.lddy = lddy; a.add = add; a.ldadd = ldadd; a.out = dx; a.ldo = lddx; a.gamma = gamma;
  a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
  a.partial = sums ? static_cast<float*>(workspace) : nullptr; a.R = R; a.F = F;
  const int64_t blocks = sum_blocks(R, F, 16 / e);
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (R > 0) {
    if (dtype == DGC_DTYPE_F32) launch<float, true>(a, blocks, st);
    else launch<uint16_t, true>(a, blocks, st);
  }
  if (sums) join_columns(a.partial, R > 0 ? blocks : 0, 2 * F, F, dgamma, dbeta, st);
  return ops::launched("norm");
}

}  // extern "C"
