// Products of rows with a weight matrix, with bias, activation and residual in the epilogue, and their gradients.
//
//   p = x w^T + bias, y = act(p) + residual          x [R, K], w [M, K], y [R, M]
//   dp = dy act'(p), dx = dp w, dw = dp^T x, dbias = sum over rows of dp
//
// One tile kernel does the three products: out[q][p] = sum over c of Q(q, c) P(p, c), where either operand's contraction
// index c lies along its rows (x, w, dp in the forward pass and in dx) or across them (w in dx; dp and x in dw).  It runs on
// v_mfma_f32_32x32x16_bf16 with P as the A operand: lane l holds outputs p = 8g + 4(l/32) + e of its own row q = l%32.
//
//  - Operand tiles are staged through registers into LDS, in units of 8 numbers along c, while the tile before is multiplied.
//    Tiles across c are read in pieces of a few columns by 8 rows and turned in registers.  A unit's place within its row
//    is rotated by the row, so that neither the fragments' reads nor the writes of turned pieces meet in a bank.
//  - bf16 numbers are taken as they are and summed in fp32.  An fp32 number is split into three bf16 parts, which hold it exactly
//    (dgc_split_dev.h), and a product is the sum of the six part products above 2^-24 of it.  The matrix unit cuts its sums off,
//    so for fp32 those of 16 terms are added up by the vector unit, which rounds: errors as of an fp32 product, 2e-7.
//  - dw is a sum over all rows with a small result: the rows are split over workgroups, each writes an fp32 partial, and a
//    second kernel adds them in order.  No atomics: the same inputs give the same bits.
//  - Up to 32 rows (a few vertices served at once) read every weight once and multiply little, and a few tiles with a long contraction
//    would keep a few compute units for long: a workgroup takes 32 x 32 outputs, its 8 waves a share of the contraction each, and
//    fragments come straight from memory.
#include <algorithm>

#include "dgc_join.h"
#include "dgc_ops.h"
#include "dgc_split_dev.h"

namespace dgc {
namespace {

using ops::Elem;
using split::as_frag;
using split::bf16x8;
using split::floatx16;

constexpr int kMaxDim = 65536;      // K, M
constexpr int kFewRows = 32;
constexpr int64_t kFewLong = 256, kFewTiles = 64;   // contraction at least, tiles of 64 x 64 at most
constexpr int64_t kNear = 1 << 23;        // pitches below it: a tile's rows are within 32 bits of each other
constexpr int64_t kMostTiles = 1 << 20;   // workgroups of one launch; more tiles are taken in turns
constexpr int64_t kRowTiles = 16;         // tiles of 32 rows that a wave takes in turn (8: 514 us, 16: 512, 4: 536 for 800 000 rows 128 -> 512)
constexpr int kSplitBlocks = 512;  // workgroups that dw is split over, about
constexpr int kSplitRows = 512;     // rows of a share of dw at least
constexpr int kSumBlocks = 1024, kMostSums = 512;   // as for the norm's weight gradients

// Whether dp takes two parts (at two_parts).  act: an activation, plus DGC_LINEAR_EXACT where the caller asks for them.
bool parted(int32_t dtype, int32_t act) {
  return dtype == DGC_DTYPE_BF16 && (act == DGC_LINEAR_EXACT + DGC_LINEAR_GELU || act == DGC_LINEAR_EXACT + DGC_LINEAR_SILU);
}
int32_t activation_of(int32_t act) { return act >= DGC_LINEAR_EXACT ? act - DGC_LINEAR_EXACT : act; }

// ---------------------------------------------------------------------------------------------- activations
// erfc(z) exp(z^2) for z >= 0 as t times a polynomial of t = 1 / (1 + 0.38 z), fitted so that the largest relative error over z in [0, 14] is
// least: 1.0e-6, 1.4e-6 in fp32.  Relative, since GELU far below zero is this tail and little else.  A fifth of the library call's
// instructions, which took longer than the memory traffic of a wide layer.
__device__ __forceinline__ float erfc_scaled(float z) {
  const float t = __builtin_amdgcn_rcpf(fmaf(0.38f, z, 1.f));
  float s = fmaf(-0.12546061f, t, 0.33618650f);
  s = fmaf(s, t, -0.07012010f);
  s = fmaf(s, t, 0.24797721f);
  s = fmaf(s, t, 0.18054272f);
  s = fmaf(s, t, 0.21658659f);
  return fmaf(s, t, 0.21428668f) * t;
}
constexpr float kRootHalf = 0.70710678118654752f, kInvRoot2Pi = 0.39894228040143268f, kLog2e = 1.4426950408889634f;

template <class T>
__device__ __forceinline__ float normal_below(float p, float& density) {   // P(X <= p), and exp(-p^2 / 2)
  if constexpr (sizeof(T) == 4) {
    density = expf(-0.5f * p * p);
    return 0.5f * erfcf(-p * kRootHalf);
  } else {
    density = __builtin_amdgcn_exp2f(-0.5f * kLog2e * p * p);
    const float tail = 0.5f * erfc_scaled(fabsf(p) * kRootHalf) * density;
    return p < 0.f ? tail : 1.f - tail;
  }
}
template <class T>
__device__ __forceinline__ float logistic(float p) {
  if constexpr (sizeof(T) == 4) return 1.f / (1.f + expf(-p));
  else return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-kLog2e * p));
}
template <class T>
__device__ __forceinline__ float activate(float p, int act) {
  float e;
  if (act == DGC_LINEAR_RELU) return p <= 0.f ? 0.f : p;     // a NaN stays one
  if (act == DGC_LINEAR_GELU) return p * normal_below<T>(p, e);
  if (act == DGC_LINEAR_SILU) return p * logistic<T>(p);
  return p;
}
template <class T>
__device__ __forceinline__ float slope_times(float dy, float p, int act) {
  if (act == DGC_LINEAR_RELU) return p <= 0.f ? 0.f : dy;
  if (act == DGC_LINEAR_GELU) {
    float e;
    const float below = normal_below<T>(p, e);
    return dy * fmaf(p * kInvRoot2Pi, e, below);
  }
  if (act == DGC_LINEAR_SILU) {
    const float s = logistic<T>(p);
    return dy * s * fmaf(p, 1.f - s, 1.f);
  }
  return dy;
}

// ---------------------------------------------------------------------------------------------- operands

template <class T> struct Kind;
template <> struct Kind<uint16_t> { static constexpr int kBK = 64, kParts = 1; };
template <> struct Kind<float> { static constexpr int kBK = 32, kParts = 3; };

// The unit of 8 numbers `u` of tile row r: its place in LDS.
template <int UK>
__device__ __forceinline__ int place(int r, int u) {
  if constexpr (UK == 8) return r * 8 + (u ^ ((r + (r >> 3)) & 7));
  else return r * 4 + (u ^ (((r >> 1) + (r >> 3)) & 3));
}
__device__ __forceinline__ void put_unit(uint4* lds, int, int at, const uint4& u) { lds[at] = u; }
__device__ __forceinline__ void put_unit(uint4* lds, int stride, int at, const float (&x)[8]) {
  uint4 p[3];
  split::split8(x, p);
#pragma unroll
  for (int q = 0; q < 3; ++q) lds[q * stride + at] = p[q];
}

// Eight numbers along the contraction from `k` of row `p`; from K on they are zero (a pitch's padding may hold anything).
__device__ __forceinline__ void load_unit(const uint16_t* p, int64_t k, int64_t K, uint4& u) {
  u = *reinterpret_cast<const uint4*>(p + k);
  if (k + 8 > K) {
    uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] &= (k + 2 * i < K ? 0xffffu : 0u) | (k + 2 * i + 1 < K ? 0xffff0000u : 0u);
    u = make_uint4(w[0], w[1], w[2], w[3]);
  }
}
__device__ __forceinline__ void load_unit(const float* p, int64_t k, int64_t K, float (&x)[8]) {
  ops::load_vec(p + k, 0, (int)min((int64_t)8, K - k), x);
  ops::load_vec(p + k, 4, (int)min((int64_t)8, K - k), x + 4);
}
__device__ __forceinline__ void take_unit(const char* p, uint4& u) { u = *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ void take_unit(const char* p, float (&x)[8]) {
  Elem<float>::unpack(reinterpret_cast<const uint4*>(p)[0], x);
  Elem<float>::unpack(reinterpret_cast<const uint4*>(p)[1], x + 4);
}
__device__ __forceinline__ void gather_unit(const uint16_t (&x)[8], uint4& u) {
  u = make_uint4(x[0] | (uint32_t)x[1] << 16, x[2] | (uint32_t)x[3] << 16, x[4] | (uint32_t)x[5] << 16, x[6] | (uint32_t)x[7] << 16);
}
__device__ __forceinline__ void gather_unit(const float (&x)[8], float (&u)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) u[i] = x[i];
}
__device__ __forceinline__ void zero_unit(uint4& u) { u = make_uint4(0, 0, 0, 0); }
__device__ __forceinline__ void zero_unit(float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = 0.f;
}
template <class T> struct UnitOf { typedef uint4 type; };
template <> struct UnitOf<float> { typedef float type[8]; };

// A tile of BX rows (of P or Q) by kBK of the contraction on its way from memory to LDS, by 256 threads.
template <class T, int BX, bool ACROSS> struct Stage;

template <class T, int BX> struct Stage<T, BX, false> {   // the contraction lies along the tensor's rows
  static constexpr int BK = Kind<T>::kBK, UK = BK / 8, N = BX * UK / 256;
  typename UnitOf<T>::type unit[N];
  __device__ __forceinline__ void load(const T* base, int64_t ld, int64_t x0, int64_t X, int64_t k0, int64_t K) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int idx = threadIdx.x + 256 * i;
      const int64_t x = x0 + idx / UK, k = k0 + idx % UK * 8;
      if (x < X && k < K) load_unit(base + x * ld, k, K, unit[i]);
      else zero_unit(unit[i]);
    }
  }
  // A tile that lies inside the tensor: a 32-bit offset for each lane from addresses that are the same for all.
  __device__ __forceinline__ void load_whole(const T* base, int64_t ld, int64_t x0, int64_t k0) {
    const uint32_t off = (threadIdx.x / UK * (uint32_t)ld + threadIdx.x % UK * 8) * sizeof(T);
#pragma unroll
    for (int i = 0; i < N; ++i) take_unit(reinterpret_cast<const char*>(base + (x0 + i * (256 / UK)) * ld + k0) + off, unit[i]);
  }
  __device__ __forceinline__ void store(uint4* lds) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int idx = threadIdx.x + 256 * i;
      put_unit(lds, BX * UK, place<UK>(idx / UK, idx % UK), unit[i]);
    }
  }
};

template <class T, int BX> struct Stage<T, BX, true> {    // the contraction goes from row to row: pieces of W columns by 8 rows
  static constexpr int BK = Kind<T>::kBK, UK = BK / 8, W = BX * UK / 256, WORDS = W * (int)sizeof(T) / 4;
  uint32_t piece[8][WORDS];
  __device__ __forceinline__ void load(const T* base, int64_t ld, int64_t x0, int64_t X, int64_t k0, int64_t K) {
    const int64_t x = x0 + threadIdx.x % (BX / W) * W, k = k0 + threadIdx.x / (BX / W) * 8;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      // a piece with a column below X lies within the pitch; its columns from X on reach no output that is kept
      const bool in = x < X && k + j < K;
      const T* at = base + (k + j) * ld + x;
      if constexpr (WORDS == 2) {
        const uint2 v = in ? *reinterpret_cast<const uint2*>(at) : make_uint2(0, 0);
        piece[j][0] = v.x; piece[j][1] = v.y;
      } else {
        piece[j][0] = in ? *reinterpret_cast<const uint32_t*>(at) : 0u;
      }
    }
  }
  __device__ __forceinline__ void store(uint4* lds) const {
    const int row = threadIdx.x % (BX / W) * W, u = threadIdx.x / (BX / W);
#pragma unroll
    for (int w = 0; w < W; ++w) {
      if constexpr (sizeof(T) == 2) {
        const uint32_t sel = w & 1 ? 0x07060302u : 0x05040100u;   // the upper or lower halves of two words
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = __builtin_amdgcn_perm(piece[2 * i + 1][w / 2], piece[2 * i][w / 2], sel);
        put_unit(lds, BX * UK, place<UK>(row + w, u), make_uint4(o[0], o[1], o[2], o[3]));
      } else {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(piece[j][w]);
        put_unit(lds, BX * UK, place<UK>(row + w, u), x);
      }
    }
  }
};

// (The second way to read a tile pays for units along the rows; for pieces across them it takes more registers than there are.)
template <class T, int BX>
__device__ __forceinline__ void fetch_stage(Stage<T, BX, false>& s, const T* base, int64_t ld, int64_t x0, int64_t X, int64_t k0, int64_t K) {
  if (k0 + Stage<T, BX, false>::BK <= K && x0 + BX <= X && ld < kNear) s.load_whole(base, ld, x0, k0);
  else s.load(base, ld, x0, X, k0, K);
}
template <class T, int BX>
__device__ __forceinline__ void fetch_stage(Stage<T, BX, true>& s, const T* base, int64_t ld, int64_t x0, int64_t X, int64_t k0, int64_t K) {
  s.load(base, ld, x0, X, k0, K);
}

// ---------------------------------------------------------------------------------------------- the tile kernel

struct LinearArgs {
  const void* P; int64_t ldp; int64_t NP;   // NP columns of the output
  const void* Q; int64_t ldq; int64_t NQ;   // NQ rows of it
  int64_t q_low;                            // two parts: where Q's low part lies, elements from Q (0: Q is as it is)
  int64_t C;                                // contraction
  int64_t share;                            // contraction of one part (a multiple of kBK); parts > 1: partial sums
  int32_t parts;
  int32_t act;
  void* out; int64_t ldo;
  const float* bias;
  const void* residual; int64_t ldr;
  void* pre; int64_t ldpre;
  float* partial;                           // [parts][NQ][NP rounded up to 4]
};

// N numbers of a row from column `col` (a multiple of N) on, 4 or 8 of them; nothing is read or written from column F on but
// what a vector of the pitch brings along.
template <class T, int N>
__device__ __forceinline__ void load_n(const T* row, int64_t col, int64_t F, float (&x)[N]) {
  const int left = (int)min((int64_t)N, F - col);
  if constexpr (N * sizeof(T) >= 16) {
#pragma unroll
    for (int i = 0; i < N; i += Elem<T>::kPer) ops::load_vec(row + col, i, left, x + i);
  } else {
    const uint2 u = *reinterpret_cast<const uint2*>(row + col);
    x[0] = split::bf_lo(u.x); x[1] = split::bf_hi(u.x); x[2] = split::bf_lo(u.y); x[3] = split::bf_hi(u.y);
  }
}
template <class T, int N>
__device__ __forceinline__ void store_n(T* row, int64_t col, int64_t F, const float (&x)[N]) {
  const int left = (int)min((int64_t)N, F - col);
  if constexpr (N * sizeof(T) >= 16) {
#pragma unroll
    for (int i = 0; i < N; i += Elem<T>::kPer) ops::store_vec(row + col, i, left, x + i);
  } else if (left >= 4) {
    *reinterpret_cast<uint2*>(row + col) = make_uint2(Elem<uint16_t>::pack2(x[0], x[1]), Elem<uint16_t>::pack2(x[2], x[3]));
  } else {
#pragma unroll
    for (int i = 0; i < 3; ++i) { if (i < left) row[col + i] = Elem<T>::one(x[i]); }
  }
}
// N outputs of row q from column p on: bias, pre-activation, activation, residual.
template <class T, int N>
__device__ __forceinline__ void finish(const LinearArgs& a, int64_t q, int64_t p, const float (&bias)[N], float (&v)[N]) {
  if (a.bias) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += bias[i];
  }
  if (a.pre) store_n<T, N>(static_cast<T*>(a.pre) + q * a.ldpre, p, a.NP, v);
  if (a.act != DGC_LINEAR_NONE) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = activate<T>(v[i], a.act);
  }
  if (a.residual) {
    float x[N];
    load_n<T, N>(static_cast<const T*>(a.residual) + q * a.ldr, p, a.NP, x);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += x[i];
  }
  store_n<T, N>(static_cast<T*>(a.out) + q * a.ldo, p, a.NP, v);
}
// The same for eight outputs inside the tensor: row q + r, column p + c, q and p the same for all lanes.
template <class T>
__device__ __forceinline__ void finish_whole(const LinearArgs& a, int64_t q, uint32_t r, int64_t p, uint32_t c, const float (&bias)[8], float (&v)[8]) {
  auto place = [&](auto* base, int64_t ld) { return base + q * ld + p + (r * (uint32_t)ld + c); };
  auto store = [&](void* base, int64_t ld) {
    T* to = place(static_cast<T*>(base), ld);
#pragma unroll
    for (int i = 0; i < 8; i += Elem<T>::kPer) *reinterpret_cast<uint4*>(to + i) = Elem<T>::pack(v + i);
  };
  if (a.bias) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += bias[i];
  }
  if (a.pre) store(a.pre, a.ldpre);
  if (a.act != DGC_LINEAR_NONE) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = activate<T>(v[i], a.act);
  }
  if (a.residual) {
    const T* from = place(static_cast<const T*>(a.residual), a.ldr);
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; i += Elem<T>::kPer) Elem<T>::unpack(*reinterpret_cast<const uint4*>(from + i), x + i);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] += x[i];
  }
  store(a.out, a.ldo);
}
template <int N>
__device__ __forceinline__ void load_bias(const LinearArgs& a, int64_t p, float (&bias)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) bias[i] = a.bias && p + i < a.NP ? a.bias[p + i] : 0.f;
}

// BP x BQ outputs a workgroup, a quarter of them a wave.  Measured: bf16 8192 x 4096 x 4096 355 to 390 us (740 TFLOP/s), fp32 8192 x 2048 x
// 2048 417 us (165 of its own, 990 of the part products); one tile's loads, products and epilogue follow each other, and two
// workgroups a CU (registers) cover part of that.
template <class T, int BP, int BQ, bool ACROSS_P, bool ACROSS_Q, bool PARTIAL, bool LOW>
__global__ __launch_bounds__(256, BP == 64 ? 3 : 2) void k_linear(LinearArgs a) {
  constexpr int BK = Kind<T>::kBK, UK = BK / 8, PARTS = Kind<T>::kParts, FP = BP / 64, FQ = BQ / 64;
  __shared__ uint4 lds[PARTS * (BP + BQ) * UK];
  uint4 *lds_p = lds, *lds_q = lds + PARTS * BP * UK;
  static_assert(BQ / 2 * BP / 4 <= PARTS * (BP + BQ) * UK, "half of the outputs fit where the operands were");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
  const int wp = (wave & 1) * (BP / 2), wq = (wave >> 1) * (BQ / 2);
  const int64_t np = (a.NP + BP - 1) / BP, nq = (a.NQ + BQ - 1) / BQ, tiles = np * nq * a.parts;
  // Workgroups go round the 8 XCDs: neighbours in the list of tiles, which share rows of Q, stay on one of them and its L2.
  const int64_t per = (tiles + 7) / 8;
  struct Tile { int64_t p0, q0, c0, c1; int part; };
  auto tile_of = [&](int64_t local) {
    const int64_t id = (int64_t)(blockIdx.x & 7) * per + local;
    Tile t;
    t.part = local < per && id < tiles ? (int)(id / (np * nq)) : -1;      // none left: -1
    t.p0 = id % np * BP;
    t.q0 = id / np % nq * BQ;
    t.c0 = (int64_t)t.part * a.share;
    t.c1 = min(a.C, t.c0 + a.share);
    return t;
  };
  const T* P = static_cast<const T*>(a.P);
  const T* Q = static_cast<const T*>(a.Q);
  Stage<T, BP, ACROSS_P> sp;
  Stage<T, BQ, ACROSS_Q> sq;
  auto fetch_p = [&](const Tile& t, int64_t c) { fetch_stage(sp, P, a.ldp, t.p0, a.NP, c, t.c1); };
  auto fetch_q = [&](const Tile& t, int64_t c, bool low) { fetch_stage(sq, LOW && low ? Q + a.q_low : Q, a.ldq, t.q0, a.NQ, c, t.c1); };
  for (int64_t local = blockIdx.x >> 3; local < per; local += gridDim.x >> 3) {
    const Tile tile = tile_of(local);
    if (tile.part < 0) return;
    fetch_p(tile, tile.c0);
    fetch_q(tile, tile.c0, true);
    const int64_t p0 = tile.p0, q0 = tile.q0, c0 = tile.c0, c1 = tile.c1;
    const int part = tile.part;
    floatx16 acc[FP][FQ];
#pragma unroll
    for (int i = 0; i < FP; ++i) {
#pragma unroll
      for (int j = 0; j < FQ; ++j) acc[i][j] = floatx16{};
    }
    auto multiply = [&]() {
      if constexpr (PARTS == 1) {
#pragma unroll
        for (int s = 0; s < BK / 16; ++s) {
          bf16x8 fp[FP], fq[FQ];
#pragma unroll
          for (int i = 0; i < FP; ++i) fp[i] = as_frag(lds_p[place<UK>(wp + 32 * i + (lane & 31), 2 * s + half)]);
#pragma unroll
          for (int j = 0; j < FQ; ++j) fq[j] = as_frag(lds_q[place<UK>(wq + 32 * j + (lane & 31), 2 * s + half)]);
#pragma unroll
          for (int i = 0; i < FP; ++i) {
#pragma unroll
            for (int j = 0; j < FQ; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp[i], fq[j], acc[i][j], 0, 0, 0);
          }
        }
      } else {
#pragma unroll
        for (int s = 0; s < BK / 16; ++s) {
          uint4 fp[FP][3], fq[FQ][3];
#pragma unroll
          for (int k = 0; k < 3; ++k) {
#pragma unroll
            for (int i = 0; i < FP; ++i) fp[i][k] = lds_p[k * BP * UK + place<UK>(wp + 32 * i + (lane & 31), 2 * s + half)];
#pragma unroll
            for (int j = 0; j < FQ; ++j) fq[j][k] = lds_q[k * BQ * UK + place<UK>(wq + 32 * j + (lane & 31), 2 * s + half)];
          }
#pragma unroll
          for (int i = 0; i < FP; ++i) {
#pragma unroll
            for (int j = 0; j < FQ; ++j) {
              floatx16 sum = {};
              split::six(sum, sum, fp[i], fq[j]);
              acc[i][j] += sum;
            }
          }
        }
      }
    };
    for (int64_t c = c0; c < c1; c += BK) {
      if constexpr (LOW) {      // Q's low part over the same tile of P first
        __syncthreads();
        sp.store(lds_p);
        sq.store(lds_q);
        __syncthreads();
        fetch_q(tile, c, false);
        multiply();
      }
      __syncthreads();
      if constexpr (!LOW) sp.store(lds_p);
      sq.store(lds_q);
      __syncthreads();
      if (c + BK < c1) {
        fetch_p(tile, c + BK);
        fetch_q(tile, c + BK, true);
      }
      multiply();
    }
    // Outputs go through LDS, half of the rows at a time, so that 16 or 8 threads finish a row's columns side by side: stored from
    // the registers as they are, each instruction touched 32 rows and the stores took longer than the products.
    constexpr int UR = BP / 4, CG = BP / 8, PASS = 256 / CG;     // 16-byte units of a row of sums; threads a row; rows at a time
    const int col = threadIdx.x % CG * 8;
    float bias[8];
    load_bias(a, p0 + col, bias);
    const bool whole = p0 + BP <= a.NP && q0 + BQ <= a.NQ && (PARTIAL ? a.NP % 4 == 0 : a.ldo < kNear && a.ldr < kNear && a.ldpre < kNear);
#pragma unroll
    for (int ph = 0; ph < 2; ++ph) {
      __syncthreads();
      if ((wave >> 1) == ph) {
#pragma unroll
        for (int j = 0; j < FQ; ++j) {
          const int row = 32 * j + (lane & 31);
#pragma unroll
          for (int i = 0; i < FP; ++i) {
#pragma unroll
            for (int g = 0; g < 4; ++g) {
              const int u = (wp + 32 * i + 8 * g + 4 * half) / 4;
              const float v[4] = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
              lds[row * UR + (u ^ (row & (UR - 1)))] = Elem<float>::pack(v);
            }
          }
        }
      }
      __syncthreads();
#pragma unroll
      for (int k = 0; k < BQ / 2 / PASS; ++k) {
        const int row = k * PASS + threadIdx.x / CG;
        const int64_t q = q0 + ph * (BQ / 2) + row, p = p0 + col;
        float v[8];
        Elem<float>::unpack(lds[row * UR + (col / 4 ^ (row & (UR - 1)))], v);
        Elem<float>::unpack(lds[row * UR + ((col / 4 + 1) ^ (row & (UR - 1)))], v + 4);
        if (whole) {
          if constexpr (PARTIAL) {
            float* to = a.partial + ((int64_t)part * a.NQ + q0 + ph * (BQ / 2) + k * PASS) * a.NP + p0;
            to += threadIdx.x / CG * (uint32_t)a.NP + col;
            *reinterpret_cast<uint4*>(to) = Elem<float>::pack(v);
            *reinterpret_cast<uint4*>(to + 4) = Elem<float>::pack(v + 4);
          } else {
            finish_whole<T>(a, q0 + ph * (BQ / 2) + k * PASS, threadIdx.x / CG, p0, col, bias, v);
          }
        } else if (q < a.NQ && p < a.NP) {
          if constexpr (PARTIAL) {
            const int64_t pitch = (a.NP + 3) / 4 * 4;
            store_n<float, 8>(a.partial + ((int64_t)part * a.NQ + q) * pitch, p, pitch, v);
          } else {
            finish<T, 8>(a, q, p, bias, v);
          }
        }
      }
    }
  }
}

// bf16 rows of 16 KF numbers, short enough for the weights to stay in registers: a wave holds 64 columns of them and takes 32 rows after
// 32 rows, which it reads as fragments straight from memory.  No wave waits for another, so products, epilogue and traffic of
// different waves overlap.  800 000 rows 128 -> 512 with GELU and the pre-activation 513 us (the tile kernel: 720), with neither 335: at
// three waves a SIMD (the weights' registers) a wave's own chain of loads, products, LDS and stores, at 3.1 to 3.6 TB/s.
template <int KF>
__global__ __launch_bounds__(256, KF <= 4 ? 4 : 3) void k_linear_rows(LinearArgs a) {
  typedef uint16_t T;
  constexpr int UR = 16;                     // 16-byte units of a row of 64 sums
  __shared__ uint4 lds[4][32 * UR];
  const int lane = threadIdx.x & 63, half = lane >> 5, tok = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  uint4* mine = lds[wave];
  // workgroups go round the 8 XCDs: those that read the same rows stay on one
  const uint32_t group = gridDim.x / 8, block = blockIdx.x < group * 8 ? blockIdx.x % 8 * group + blockIdx.x / 8 : blockIdx.x;
  const uint32_t line = block * 4 + wave, across = (uint32_t)(a.NP / 64), tiles = (uint32_t)((a.NQ + 31) / 32);
  const int64_t p0 = (int64_t)(line % across) * 64;
  uint32_t tile = line / across * (uint32_t)a.share;
  const uint32_t end = min(tiles, tile + (uint32_t)a.share);
  if (tile >= tiles) return;
  const T* Q = static_cast<const T*>(a.Q);
  bf16x8 fp[2][KF];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const T* P = static_cast<const T*>(a.P) + (p0 + 32 * i) * a.ldp + (tok * (uint32_t)a.ldp + 8 * half);
#pragma unroll
    for (int k = 0; k < KF; ++k) fp[i][k] = as_frag(*reinterpret_cast<const uint4*>(P + 16 * k));
  }
  const uint32_t col = lane % 8 * 8;
  float bias[8];
  load_bias(a, p0 + col, bias);
  uint4 raw[KF];
  auto fetch = [&](uint32_t t) {
    const uint32_t r = min((uint32_t)tok, (uint32_t)min(a.NQ - 1 - (int64_t)t * 32, (int64_t)31));  // rows behind the last are not kept
    const T* row = Q + (int64_t)t * 32 * a.ldq + (r * (uint32_t)a.ldq + 8 * half);
#pragma unroll
    for (int k = 0; k < KF; ++k) raw[k] = *reinterpret_cast<const uint4*>(row + 16 * k);
  };
  fetch(tile);
  for (; tile < end; ++tile) {
    floatx16 acc[2] = {};
#pragma unroll
    for (int k = 0; k < KF; ++k) {
#pragma unroll
      for (int i = 0; i < 2; ++i) acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fp[i][k], as_frag(raw[k]), acc[i], 0, 0, 0);
    }
    if (tile + 1 < end) fetch(tile + 1);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float v[4] = {acc[i][4 * g], acc[i][4 * g + 1], acc[i][4 * g + 2], acc[i][4 * g + 3]};
        mine[tok * UR + ((8 * i + 2 * g + half) ^ (tok & 15))] = Elem<float>::pack(v);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll 1
    for (int k = 0; k < 4; ++k) {
      const int row = 8 * k + lane / 8;
      float v[8];
      Elem<float>::unpack(mine[row * UR + (col / 4 ^ (row & 15))], v);
      Elem<float>::unpack(mine[row * UR + ((col / 4 + 1) ^ (row & 15))], v + 4);
      if ((int64_t)tile * 32 + row < a.NQ) finish_whole<T>(a, (int64_t)tile * 32 + 8 * k, lane / 8, p0, col, bias, v);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// Few outputs, or few rows: 32 rows by 32 columns a workgroup, 8 waves that take 64 of the contraction at a time in turn.  8 rows 1024 -> 4096:
// 6 us, one round of loads and the join; 8 MB of weights are 1.7 us.
template <class T, bool ACROSS_P, bool LOW>
__global__ __launch_bounds__(512) void k_linear_few(LinearArgs a) {
  __shared__ float joined[8][16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
  const int64_t p0 = (int64_t)blockIdx.x * 32, p = p0 + (lane & 31), q = (int64_t)blockIdx.y * 32 + (lane & 31);
  const T* P = static_cast<const T*>(a.P) + (ACROSS_P ? p : p * a.ldp);
  const T* Q = static_cast<const T*>(a.Q) + q * a.ldq;
  floatx16 acc = floatx16{};
  for (int64_t c = wave * 64; c < a.C; c += 8 * 64) {
    typename UnitOf<T>::type up[4], uq[4], ul[LOW ? 4 : 1];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int64_t k = c + 16 * s + 8 * half;
      if constexpr (ACROSS_P) {
        T x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = p < a.NP && k + e < a.C ? P[(k + e) * a.ldp] : T(0);
        gather_unit(x, up[s]);
      } else {
        if (p < a.NP && k < a.C) load_unit(P, k, a.C, up[s]);
        else zero_unit(up[s]);
      }
      if (q < a.NQ && k < a.C) load_unit(Q, k, a.C, uq[s]);
      else zero_unit(uq[s]);
      if constexpr (LOW) {
        if (q < a.NQ && k < a.C) load_unit(Q + a.q_low, k, a.C, ul[s]);
        else zero_unit(ul[s]);
      }
    }
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        if constexpr (LOW) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_frag(up[s]), as_frag(ul[s]), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_frag(up[s]), as_frag(uq[s]), acc, 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        uint4 fp[3], fq[3];
        split::split8(up[s], fp);
        split::split8(uq[s], fq);
        floatx16 sum = floatx16{};
        split::six(sum, sum, fp, fq);
        acc += sum;
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) joined[wave][i][lane] = acc[i];
  __syncthreads();
  // a thread finishes four columns of a row: register 4 g + e of lane (row, half) is column 8 g + 4 half + e
  if (threadIdx.x < 256) {
    const int g = threadIdx.x >> 6;
    const int64_t col = p0 + 8 * g + 4 * half;
    float v[4] = {};
#pragma unroll
    for (int w = 0; w < 8; ++w) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] += joined[w][4 * g + e][lane];
    }
    if (q < a.NQ && col < a.NP) {
      float bias[4];
      load_bias(a, col, bias);
      finish<T, 4>(a, q, col, bias, v);
    }
  }
}

// The partial sums of dw: 16 units of four columns a workgroup, 16 parts at a time (512 x 128 from 128 parts: 7 us).
template <class T>
__global__ __launch_bounds__(256) void k_linear_join(LinearArgs a) {
  __shared__ float4 lds[16][16];
  const int c = threadIdx.x & 15, g = threadIdx.x >> 4;
  const int64_t pitch = (a.NP + 3) / 4, n = a.NQ * pitch, unit = (int64_t)blockIdx.x * 16 + c;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  if (unit < n) {
#pragma unroll 4
    for (int part = g; part < a.parts; part += 16) {
      const float4 x = *reinterpret_cast<const float4*>(a.partial + (part * n + unit) * 4);
      v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
    }
  }
  lds[g][c] = v;
  __syncthreads();
#pragma unroll
  for (int m = 8; m >= 1; m >>= 1) {
    if (g < m) {
      const float4 x = lds[g + m][c];
      v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
      lds[g][c] = v;
    }
    __syncthreads();
  }
  if (g == 0 && unit < n) {
    float y[4] = {v.x, v.y, v.z, v.w};
    const float none[4] = {};
    finish<T, 4>(a, unit / pitch, unit % pitch * 4, none, y);
  }
}

// ---------------------------------------------------------------------------------------------- dp and dbias

struct SlopeArgs {
  const void* dy; int64_t lddy;
  const void* pre; int64_t ldpre;
  void* dp; int64_t lddp;        // nullptr: act is none, dp is dy itself
  int64_t low;                   // two parts: where the low one lies, elements from dp (0: one part)
  float* partial;                // [workgroups][M], or nullptr
  int64_t R;
  int32_t M;
  int32_t act;
};

// The matrix unit takes bf16.  dp rounded to one such number, 2^-8, adds as much to the error of dx and dw as their own rounding does
// (2.3e-3 of their norm for 1.7e-3), and is what a training step in bf16 takes by default: in two parts, 2^-16, dp is twice the traffic and the products are
// twice the matrix work (400 000 rows 128 -> 512 with GELU 510 us and 915, 8192 rows 4096 -> 4096 810 us and 1430).  So that is the caller's
// choice, DGC_LINEAR_EXACT, for GELU and SILU: RELU's dp is dy or 0, one bf16 number.  Both parts have dp's sign, the high one by cutting off
// and the low one by never being zero where dp (from 2^-109 on) is not, so that dp times an infinity is that infinity.
__device__ __forceinline__ void two_parts(float dp, float& high, float& low) {
  high = dp == dp ? split::cut(dp) : dp;
  const float rest = dp - high;
  low = fabsf(rest) >= 0x1p-126f || fabsf(dp) < 0x1p-109f ? rest : copysignf(0x1p-126f, dp);
}

// 400 000 x 512 bf16 with GELU: 245 us, 5 TB/s of dy, pre and dp.  LPR lanes a row, 256 / LPR rows at a time; blockIdx.y: which LPR vectors of a wide row.
template <class T, int LPR, bool LOW>
__global__ __launch_bounds__(256) void k_linear_slope(SlopeArgs a) {
  constexpr int VN = Elem<T>::kPer, GROUPS = 256 / LPR, U = 4;
  __shared__ float joined[256 * VN];
  const int sub = threadIdx.x % LPR, grp = threadIdx.x / LPR;
  const int col = ((int)blockIdx.y * LPR + sub) * VN;
  float sum[VN] = {};
  for (int64_t base = (int64_t)blockIdx.x * (GROUPS * U); base < a.R; base += (int64_t)gridDim.x * (GROUPS * U)) {
    float dy[U][VN], p[U][VN];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t r = base + u * GROUPS + grp;
      ops::load_vec(static_cast<const T*>(a.dy) + r * a.lddy, col, r < a.R ? a.M : 0, dy[u]);
      if (a.dp) ops::load_vec(static_cast<const T*>(a.pre) + r * a.ldpre, col, r < a.R ? a.M : 0, p[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int64_t r = base + u * GROUPS + grp;
      if (a.dp) {
#pragma unroll
        for (int i = 0; i < VN; ++i) dy[u][i] = slope_times<T>(dy[u][i], p[u][i], a.act);
        if (r < a.R && col < a.M) {
          T* to = static_cast<T*>(a.dp) + r * a.lddp + col;
          if constexpr (LOW) {
            float high[VN], low[VN];
#pragma unroll
            for (int i = 0; i < VN; ++i) two_parts(dy[u][i], high[i], low[i]);
            *reinterpret_cast<uint4*>(to) = Elem<T>::pack(high);
            *reinterpret_cast<uint4*>(to + a.low) = Elem<T>::pack(low);
          } else {
            *reinterpret_cast<uint4*>(to) = Elem<T>::pack(dy[u]);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < VN; ++i) sum[i] += dy[u][i];
    }
  }
  if (!a.partial) return;
#pragma unroll
  for (int i = 0; i < VN; ++i) joined[threadIdx.x * VN + i] = sum[i];
  __syncthreads();
  for (int c = threadIdx.x; c < LPR * VN; c += 256) {
    const int64_t m = (int64_t)blockIdx.y * LPR * VN + c;
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < GROUPS; ++k) s += joined[k * LPR * VN + c];
    if (m < a.M) a.partial[(int64_t)blockIdx.x * a.M + m] = s;
  }
}

int slope_lanes(int32_t M, int per) {
  const int vecs = (M + per - 1) / per;
  int lpr = 8;
  while (lpr < vecs && lpr < 256) lpr *= 2;
  return lpr;
}
int64_t slope_blocks(int64_t R, int32_t M, int per) {
  const int64_t rows = 256 / slope_lanes(M, per) * 4, turns = (R + rows - 1) / rows;
  const int64_t wide = ((M + per - 1) / per + 255) / 256;      // blockIdx.y
  return std::max<int64_t>(std::min<int64_t>(turns, std::max<int64_t>(kSumBlocks / wide, 64)), (turns * 4 + kMostSums - 1) / kMostSums);
}

template <class T, bool LOW>
void launch_slope(const SlopeArgs& a, int64_t blocks, hipStream_t st) {
  const int per = Elem<T>::kPer, lpr = slope_lanes(a.M, per), vecs = (a.M + per - 1) / per;
  const dim3 grid((unsigned)blocks, (unsigned)((vecs + lpr - 1) / lpr));
  if (lpr == 8) hipLaunchKernelGGL((k_linear_slope<T, 8, LOW>), grid, 256, 0, st, a);
  else if (lpr == 16) hipLaunchKernelGGL((k_linear_slope<T, 16, LOW>), grid, 256, 0, st, a);
  else if (lpr == 32) hipLaunchKernelGGL((k_linear_slope<T, 32, LOW>), grid, 256, 0, st, a);
  else if (lpr == 64) hipLaunchKernelGGL((k_linear_slope<T, 64, LOW>), grid, 256, 0, st, a);
  else if (lpr == 128) hipLaunchKernelGGL((k_linear_slope<T, 128, LOW>), grid, 256, 0, st, a);
  else hipLaunchKernelGGL((k_linear_slope<T, 256, LOW>), grid, 256, 0, st, a);
}

// ---------------------------------------------------------------------------------------------- host

// 128 x 128 outputs a workgroup; 64 x 64 where that leaves compute units without work, or the output is that narrow.
// fp32 forward, small against large tiles, us: 100 000 rows 172 -> 128 (782 large tiles) 52, 56; 40 000 256 -> 256 (626) 49, 56; 120 000 128 -> 128 (938) 42, 43;
// 25 000 512 -> 512 (784) 113, 106.  fp32 dx, where a tile's weights are turned and split, too, so that small tiles repeat more: 60 001 256 -> 256 (938) 85, 72; 25 000
// 512 -> 512 (784) 134, 114; 120 000 128 -> 128 (938) 50, 46; 40 000 256 -> 256 (626) 58, 62; 4000 1024 -> 1024 (256) 101, 92.
template <class T, bool ACROSS_P>
bool small_tiles(int64_t NP, int64_t NQ) {
  return NP <= 64 || NQ <= 64 || ((NP + 127) / 128) * ((NQ + 127) / 128) < (sizeof(T) == 4 && !ACROSS_P ? 1024 : 256);
}

// Up to 32 rows, or so few tiles with so long a contraction that it is better split over the waves of more workgroups: bf16 100 x 4000 -> 50
// 12 us for 48 in tiles, 200 x 2000 -> 200 8 for 23; fp32 500 x 300 -> 500 8 for 16, 100 x 4000 -> 50 42 for 159.
bool few_outputs(int64_t NP, int64_t NQ, int64_t C) {
  return NQ <= kFewRows || (C >= kFewLong && ((NP + 63) / 64) * ((NQ + 63) / 64) <= kFewTiles);
}
template <class T, bool ACROSS_P, bool LOW>
void launch_few(const LinearArgs& a, hipStream_t st) {
  hipLaunchKernelGGL((k_linear_few<T, ACROSS_P, LOW>), dim3((unsigned)((a.NP + 31) / 32), (unsigned)((a.NQ + 31) / 32)), 512, 0, st, a);
}

template <class T, bool ACROSS_P, bool ACROSS_Q, bool PARTIAL, bool LOW>
void launch_tiles(const LinearArgs& a, bool small, hipStream_t st) {
  const int64_t b = small ? 64 : 128, tiles = ((a.NP + b - 1) / b) * ((a.NQ + b - 1) / b) * a.parts;
  const unsigned grid = (unsigned)(std::min<int64_t>((tiles + 7) / 8, kMostTiles / 8) * 8);
  if (small) hipLaunchKernelGGL((k_linear<T, 64, 64, ACROSS_P, ACROSS_Q, PARTIAL, LOW>), grid, 256, 0, st, a);
  else hipLaunchKernelGGL((k_linear<T, 128, 128, ACROSS_P, ACROSS_Q, PARTIAL, LOW>), grid, 256, 0, st, a);
}

// The kernel for short rows takes these (the largest pitch that is not there is 0).
bool short_rows(const LinearArgs& a, int32_t dtype) {
  return dtype == DGC_DTYPE_BF16 && a.C <= 128 && a.C % 32 == 0 && a.NP % 64 == 0 && (a.NQ + 31) / 32 * (a.NP / 64) < ((int64_t)1 << 31) &&
         std::max({a.ldp, a.ldq, a.ldo, a.ldr, a.ldpre}) < kNear;
}
// Tiles of 32 rows that a wave takes one after the other, enough waves to fill the chip first.
void launch_rows(LinearArgs a, hipStream_t st) {
  const int64_t across = a.NP / 64, tiles = (a.NQ + 31) / 32;
  a.share = std::max<int64_t>(1, std::min<int64_t>(kRowTiles, tiles * across / (256 * 4 * 3)));
  a.share = std::max(a.share, (tiles * across + 4 * kMostBlocks - 1) / (4 * kMostBlocks));    // grids end below 2^32 threads
  const int64_t waves = (tiles + a.share - 1) / a.share * across;
  const unsigned grid = (unsigned)((waves + 3) / 4);
  if (a.C == 32) hipLaunchKernelGGL(k_linear_rows<2>, grid, 256, 0, st, a);
  else if (a.C == 64) hipLaunchKernelGGL(k_linear_rows<4>, grid, 256, 0, st, a);
  else if (a.C == 96) hipLaunchKernelGGL(k_linear_rows<6>, grid, 256, 0, st, a);
  else hipLaunchKernelGGL(k_linear_rows<8>, grid, 256, 0, st, a);
}

// How dw's rows are split: enough shares to fill the chip, none below kSplitRows.
struct Split { bool small; int32_t parts; int64_t share; };
Split split_of(int64_t R, int64_t K, int64_t M) {
  Split s;
  s.small = K <= 64 || M <= 64;
  const int64_t b = s.small ? 64 : 128, tiles = ((K + b - 1) / b) * ((M + b - 1) / b);
  const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(kSplitBlocks / tiles, (R + kSplitRows - 1) / kSplitRows));
  s.share = std::max<int64_t>(64, ((R + parts - 1) / parts + 63) / 64 * 64);
  s.parts = (int32_t)std::max<int64_t>(1, (R + s.share - 1) / s.share);
  return s;
}

struct Room { int64_t dp, sums, partial, all; };   // where each starts in the workspace, bytes
Room room_of(int64_t R, int32_t K, int32_t M, int32_t dtype, int32_t act) {
  const int e = ops::elem_bytes(dtype), per = 16 / e;
  const Split s = split_of(R, K, M);
  Room r;
  r.dp = 0;
  r.sums = activation_of(act) == DGC_LINEAR_NONE ? 0 : R * ((M + per - 1) / per * per) * e * (parted(dtype, act) ? 2 : 1);
  r.partial = r.sums + (slope_blocks(R, M, per) * M + 3) / 4 * 16;
  r.all = r.partial + (s.parts > 1 ? 4 * (int64_t)s.parts * M * ((K + 3) / 4 * 4) : 0) + 16;
  return r;
}

// dx and dw from dp, whose low part lies `low` elements behind it (LOW).
template <class T, bool LOW>
void products(const void* dp, int64_t lddp, int64_t low, const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t R, int32_t K, int32_t M,
              void* dx, int64_t lddx, void* dw, int64_t lddw, float* partial, hipStream_t st) {
  LinearArgs a{};
  a.Q = dp; a.ldq = lddp; a.q_low = low; a.NP = K;
  if (dw) {
    const Split s = split_of(R, K, M);
    a.P = x; a.ldp = ldx; a.NQ = M; a.C = R; a.share = s.share; a.parts = s.parts;
    a.out = dw; a.ldo = lddw; a.partial = partial;
    if (s.parts == 1) {
      launch_tiles<T, true, true, false, LOW>(a, s.small, st);
    } else {
      launch_tiles<T, true, true, true, LOW>(a, s.small, st);
      const int64_t n = (int64_t)M * ((K + 3) / 4);
      hipLaunchKernelGGL(k_linear_join<T>, (unsigned)((n + 15) / 16), 256, 0, st, a);
    }
  }
  if (dx && R > 0) {
    a.P = w; a.ldp = ldw; a.NQ = R; a.C = M; a.share = (M + 63) / 64 * 64; a.parts = 1;
    a.out = dx; a.ldo = lddx; a.partial = nullptr;
    if (few_outputs(a.NP, a.NQ, a.C)) launch_few<T, true, LOW>(a, st);
    else launch_tiles<T, true, false, false, LOW>(a, small_tiles<T, true>(a.NP, a.NQ), st);
  }
}

template <class T>
void backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t R, int32_t K, int32_t M,
              const void* pre, int64_t ldpre, int32_t act, bool two, void* dx, int64_t lddx, void* dw, int64_t lddw, float* dbias,
              char* workspace, const Room& room, hipStream_t st) {
  const void* dp = dy;
  int64_t lddp = lddy, low = 0;
  const int64_t blocks = slope_blocks(R, M, Elem<T>::kPer);
  float *sums = reinterpret_cast<float*>(workspace + room.sums), *partial = reinterpret_cast<float*>(workspace + room.partial);
  if (R > 0 && (dbias || act != DGC_LINEAR_NONE)) {
    SlopeArgs s{};
    s.dy = dy; s.lddy = lddy; s.pre = pre; s.ldpre = ldpre; s.R = R; s.M = M; s.act = act;
    s.partial = dbias ? sums : nullptr;
    if (act != DGC_LINEAR_NONE) {
      s.dp = workspace + room.dp;
      s.lddp = (M + Elem<T>::kPer - 1) / Elem<T>::kPer * Elem<T>::kPer;
      if (two) {      // a row's low parts behind its high ones
        s.low = low = s.lddp;
        s.lddp *= 2;
      }
      dp = s.dp; lddp = s.lddp;
    }
    if (two && s.dp) launch_slope<T, sizeof(T) == 2>(s, blocks, st);
    else launch_slope<T, false>(s, blocks, st);
  }
  if (dbias) join_columns(sums, R > 0 ? blocks : 0, M, M, dbias, nullptr, st);
  if (two && low > 0) products<T, sizeof(T) == 2>(dp, lddp, low, x, ldx, w, ldw, R, K, M, dx, lddx, dw, lddw, partial, st);
  else products<T, false>(dp, lddp, 0, x, ldx, w, ldw, R, K, M, dx, lddx, dw, lddw, partial, st);
}

const char* check(int64_t R, int32_t K, int32_t M, int32_t dtype, int32_t act) {
  if (dtype != DGC_DTYPE_F32 && dtype != DGC_DTYPE_BF16) return "linear: unknown dtype";
  if (R < 0 || K < 1 || M < 1 || K > kMaxDim || M > kMaxDim) return "linear: R must be >= 0, K and M in [1, 65536]";
  if (R > INT64_MAX / 8 / kMaxDim) return "linear: too many rows";
  if (act < DGC_LINEAR_NONE || act > DGC_LINEAR_SILU) return "linear: unknown activation";
  return nullptr;
}

}  // namespace
}  // namespace dgc

using namespace dgc;

extern "C" {

int64_t dgc_linear_workspace_bytes(int64_t R, int32_t K, int32_t M, int32_t dtype, int32_t act) {
  if (check(R, K, M, dtype, activation_of(act))) return -1;
  return room_of(R, K, M, dtype, act).all;
}

dgc_status_t dgc_linear_forward(const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t R, int32_t K, int32_t M,
                                int32_t dtype, const float* bias, int32_t act, const void* residual, int64_t ldr, void* y,
                                int64_t ldy, void* pre, int64_t ldpre, void* stream) {
  if (const char* msg = check(R, K, M, dtype, act)) return ops::refuse(DGC_ERR_INVALID_ARG, msg);
  const int e = ops::elem_bytes(dtype);
  if (!ops::good_rows(x, R, K, ldx, e) || !ops::good_rows(w, M, K, ldw, e) || !ops::good_rows(y, R, M, ldy, e) ||
      (residual && !ops::good_rows(residual, R, M, ldr, e)) || (pre && !ops::good_rows(pre, R, M, ldpre, e)))
    return ops::refuse(DGC_ERR_INVALID_ARG, "linear: x, w, residual, y, pre need a 16-byte aligned base and a pitch that holds a row and is a multiple of 16 bytes");
  if (ops::share(x, ldx, e, K, y, ldy, e, M, R) || ops::share(x, ldx, e, K, pre, ldpre, e, M, R) ||
      ops::share(y, ldy, e, M, pre, ldpre, e, M, R) || ops::share(residual, ldr, e, M, pre, ldpre, e, M, R) ||
      (!ops::same_place(residual, ldr, y, ldy) && ops::share(residual, ldr, e, M, y, ldy, e, M, R)) ||
      ops::span_shared(w, ldw, e, K, M, y, ldy, e, M, R) || ops::span_shared(w, ldw, e, K, M, pre, ldpre, e, M, R))
    return ops::refuse(DGC_ERR_INVALID_ARG, "linear: y and pre lie apart from the inputs and each other (y may be residual itself)");
  if (R == 0) return DGC_OK;
  LinearArgs a{};
  a.P = w; a.ldp = ldw; a.NP = M; a.Q = x; a.ldq = ldx; a.NQ = R; a.C = K; a.share = (K + 63) / 64 * 64; a.parts = 1; a.act = act;
  a.out = y; a.ldo = ldy; a.bias = bias; a.residual = residual; a.ldr = ldr; a.pre = pre; a.ldpre = ldpre;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (few_outputs(M, R, K)) {
    if (dtype == DGC_DTYPE_F32) launch_few<float, false, false>(a, st);
    else launch_few<uint16_t, false, false>(a, st);
  } else if (short_rows(a, dtype)) {
    launch_rows(a, st);
  } else if (dtype == DGC_DTYPE_F32) {
    launch_tiles<float, false, false, false, false>(a, small_tiles<float, false>(M, R), st);
  } else {
    launch_tiles<uint16_t, false, false, false, false>(a, small_tiles<uint16_t, false>(M, R), st);
  }
  return ops::launched("linear");
}

dgc_status_t dgc_linear_backward(const void* dy, int64_t lddy, const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t R,
                                 int32_t K, int32_t M, int32_t dtype, const void* pre, int64_t ldpre, int32_t act, void* dx,
                                 int64_t lddx, void* dw, int64_t lddw, float* dbias, void* workspace, int64_t workspace_bytes,
                                 void* stream) {
  const bool two = parted(dtype, act);
  const int32_t f = activation_of(act);
  if (const char* msg = check(R, K, M, dtype, f)) return ops::refuse(DGC_ERR_INVALID_ARG, msg);
  const int e = ops::elem_bytes(dtype);
  const bool pre_used = f != DGC_LINEAR_NONE;
  if (!ops::good_rows(dy, R, M, lddy, e) || (dw && !ops::good_rows(x, R, K, ldx, e)) || (dx && !ops::good_rows(w, M, K, ldw, e)) ||
      (pre_used && !ops::good_rows(pre, R, M, ldpre, e)) || (dx && !ops::good_rows(dx, R, K, lddx, e)) ||
      (dw && !ops::good_rows(dw, M, K, lddw, e)))
    return ops::refuse(DGC_ERR_INVALID_ARG, "linear: dy, x, w, pre, dx, dw need a 16-byte aligned base and a pitch that holds a row and is a multiple of 16 bytes");
  if (!dw) x = nullptr;
  if (!dx) w = nullptr;
  if (!pre_used) pre = nullptr;
  if (ops::share(dx, lddx, e, K, dy, lddy, e, M, R) || ops::share(dx, lddx, e, K, x, ldx, e, K, R) ||
      ops::share(dx, lddx, e, K, pre, ldpre, e, M, R) || ops::span_shared(w, ldw, e, K, M, dx, lddx, e, K, R) ||
      ops::span_shared(dw, lddw, e, K, M, dx, lddx, e, K, R) || ops::span_shared(dw, lddw, e, K, M, dy, lddy, e, M, R) ||
      ops::span_shared(dw, lddw, e, K, M, x, ldx, e, K, R) || ops::span_shared(dw, lddw, e, K, M, pre, ldpre, e, M, R) ||
      ops::share(dw, lddw, e, K, w, ldw, e, K, M))
    return ops::refuse(DGC_ERR_INVALID_ARG, "linear: dx and dw lie apart from the inputs and each other");
  const Room room = room_of(R, K, M, dtype, act);
  if (!workspace || !ops::aligned16(workspace) || workspace_bytes < room.all)
    return ops::refuse(DGC_ERR_INVALID_ARG, "linear: workspace missing, too small (dgc_linear_workspace_bytes) or not 16-byte aligned");
  hipStream_t st = static_cast<hipStream_t>(stream);
  char* ws = static_cast<char*>(workspace);
  if (dtype == DGC_DTYPE_F32)
    backward<float>(dy, lddy, x, ldx, w, ldw, R, K, M, pre, ldpre, f, false, dx, lddx, dw, lddw, dbias, ws, room, st);
  else
    backward<uint16_t>(dy, lddy, x, ldx, w, ldw, R, K, M, pre, ldpre, f, two, dx, lddx, dw, lddw, dbias, ws, room, st);
  return ops::launched("linear");
}

}  // extern "C"
