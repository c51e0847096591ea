// Linear attention with a decay per head: a time encoder whose state is a matrix per sequence and head.
//
//   S_t = l_t g S_{t-1} + k_t^T v_t   (l_t = 0 where a reset flag is set, else 1),   o_t = s q_t S_t
//
// One kernel computes the forward pass and all gradients.  With roles A, B, C for q, k, v it is
//   out_i = alpha sum_{j <= i} g^(i-j) (A_i . B_j) C_j + gam g^(i+1) A_i S_in,   S = g^n S_in + beta sum_j g^(n-1-j) B_j^T C_j
// (sums over the tokens since the last reset, S_in only before the first), and the gradients are the same sums:
//   dq: A, B, C = do, v, k from S_0^T;   with G_t = s q_t^T do_t + l_{t+1} g G_{t+1}, walked from the last token to the first,
//   dv: A, B, C = k, q, do and dk: A, B, C = v, do, q from dS_N (not decayed) and its transpose;   dS_0 = l_0 g G_0.
//
// A wave takes 32 tokens of one sequence and head and 32 columns of C at a time and keeps its part of S in registers from one
// 32 to the next.  All products run on v_mfma_f32_32x32x16_bf16, operands and results in registers (LDS holds outputs on their way to memory,
// and in k_decay_window_back states of up to 32 x 32 on theirs from it):
//  - scores D[j][i] = B_j . A_i leave lane i with 16 scores of its own token i in just the order in which a product that sums over
//    j takes them; C, and B for the state, come into that order by a product with the identity, which is exact;
//  - the state's rows are kept in the order that makes its registers the operand of A S: row 8g + 4(l/32) + e of a tile is
//    number swap(8g + 4(l/32) + e) of B's, swap exchanging bits 2 and 3.
// Rounding: bf16 tensors enter as they are.  Scores and states, which are fp32, enter in parts: two bf16 parts (2^-17) where the
// result is rounded to bf16, three (all 24 bits) where it goes into the fp32 state; fp32 tensors always in three, six part
// products a product.  The matrix unit cuts its sums off, so the state is carried from one 32 tokens to the next by the vector unit.
// A zero score or weight times a value that is not finite would be NaN for tokens that do not see that value: 32 tokens with such
// a value go one by one.
//
// Few long sequences are split into segments: a first pass leaves each segment's own state, a scan joins them into the states
// that enter the segments, a second pass starts from those.  One token (serving a new snapshot) has a kernel of its own that
// reads and writes the states as the stream they are.  No atomics: the same inputs give the same bits.
#include <algorithm>

#include "dgc_ops.h"
#include "dgc_split_dev.h"

namespace dgc {
namespace {

using ops::Elem;
using split::as_frag;
using split::floatx16;

constexpr int kMaxHeads = 1024, kMaxDim = 128;
constexpr int kTok = 32;               // tokens at a time
constexpr int64_t kFillWaves = 2048;   // two a SIMD
constexpr int64_t kSegTokens = 128;    // tokens of a segment at least
constexpr int64_t kRun = 8;            // rows that a wave takes in turn

struct Rows {          // row (t, i) at p + t st + i sn, in elements
  const void* p;
  int64_t st, sn;
};

struct DecayArgs {
  Rows A, B, C, O;
  int64_t T, N;
  int32_t heads, dk, dv;        // dk: length of A's and B's rows, dv: of C's and O's, a head
  int32_t blocks_v;             // 32 columns of C each
  int32_t reversed;             // tokens from the last to the first
  float alpha, beta, gam;
  const float* decay;
  const uint8_t* reset;         // [T][N] or nullptr
  const int32_t* lengths;       // [N] or nullptr
  const float* s_in;            // state (i, h) [seg] element (r, c) at s_in + ((seg N + i) heads + h) dk dv + r in_r + c in_c, or nullptr
  int32_t in_r, in_c;
  float* s_out;                 // the same, or nullptr
  int32_t out_r, out_c;
  int32_t out_link;             // the state is written times l_0 g (of no token: as it came in)
  float* factor;                // first pass: what a segment keeps of the state entering it, [seg][N][heads]; -1: cut off by a reset
  int32_t segs;
  int64_t seg_len;
  uint32_t run;                 // sequences (or pairs, or segments) that a wave takes one after the other
};

// The product of operands in parts, those below 2^-24 left out, the smallest first.
template <int NX, int NY>
__device__ __forceinline__ void mul(floatx16& c, const uint4 (&x)[NX], const uint4 (&y)[NY]) {
#pragma unroll
  for (int s = 2; s >= 0; --s) {
#pragma unroll
    for (int i = 0; i <= s; ++i) {
      if (i < NX && s - i < NY) c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_frag(x[i]), as_frag(y[s - i]), c, 0, 0, 0);
    }
  }
}
template <int N>
__device__ __forceinline__ void parts_of(const float (&x)[8], uint4 (&p)[N]) {
  if constexpr (N == 3) {
    split::split8(x, p);
  } else {
    uint32_t h[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      h[i] = split::nearest(x[2 * i], x[2 * i + 1]);
      l[i] = split::nearest(x[2 * i] - split::bf_lo(h[i]), x[2 * i + 1] - split::bf_hi(h[i]));
    }
    p[0] = make_uint4(h[0], h[1], h[2], h[3]);
    if constexpr (N == 2) p[1] = make_uint4(l[0], l[1], l[2], l[3]);
  }
}

// How many parts: of a tensor's numbers, of scores and states in a product that is rounded to the tensors' type, of the state's.
template <class T> struct Kind;
template <> struct Kind<uint16_t> { static constexpr int kIn = 1, kMid = 2; };
template <> struct Kind<float> { static constexpr int kIn = 3, kMid = 3; };

template <class T> __device__ __forceinline__ float to_float(T x);
template <> __device__ __forceinline__ float to_float<float>(float x) { return x; }
template <> __device__ __forceinline__ float to_float<uint16_t>(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

__device__ __forceinline__ int swap23(int x) { return (x & ~12) | (x & 4) << 1 | (x & 8) >> 1; }
__device__ __forceinline__ uint4 identity(int c, int half, int n) {   // rows 16 c + 8 half + 0..7 of its column n
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 16 * c + 8 * half + 2 * i;
    w[i] = (r == n ? 0x3f80u : 0u) | (r + 1 == n ? 0x3f800000u : 0u);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ float power(float g, uint32_t n) {   // g^n by squaring, in double, so that far powers keep their bits
  double r = 1., x = (double)g;
  for (; n; n >>= 1) {
    if (n & 1) r *= x;
    x *= x;
  }
  return (float)r;
}
__device__ __forceinline__ void not_finite(float& t, const floatx16& x) {   // t turns NaN if one of them is not finite
#pragma unroll
  for (int r = 0; r < 16; ++r) t = fmaf(x[r], 0.f, t);
}

// Raw fragments of a row: 8 numbers from each of a lane's places, as they lie in memory.
template <class T> struct Raw8 { uint4 w[sizeof(T) == 2 ? 1 : 2]; };
template <class T>
__device__ __forceinline__ Raw8<T> fetch8(const T* p, bool in) {
  Raw8<T> r;
#pragma unroll
  for (int k = 0; k < (int)(sizeof(r) / 16); ++k) r.w[k] = in ? reinterpret_cast<const uint4*>(p)[k] : make_uint4(0, 0, 0, 0);
  return r;
}
template <class T>
__device__ __forceinline__ void operand(const Raw8<T>& r, uint4 (&f)[Kind<T>::kIn]) {
  if constexpr (sizeof(T) == 2) {
    f[0] = r.w[0];
  } else {
    float x[8];
    Elem<float>::unpack(r.w[0], x);
    Elem<float>::unpack(r.w[1], x + 4);
    split::split8(x, f);
  }
}
template <class T>
__device__ __forceinline__ void store4(T* to, const float (&x)[4]) {
  if constexpr (sizeof(T) == 4) *reinterpret_cast<uint4*>(to) = Elem<float>::pack(x);
  else *reinterpret_cast<uint2*>(to) = make_uint2(Elem<uint16_t>::pack2(x[0], x[1]), Elem<uint16_t>::pack2(x[2], x[3]));
}
template <int N>
__device__ __forceinline__ void half_parts(const floatx16& x, int k, uint4 (&p)[N]) {   // registers 8 k .. 8 k + 7
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = x[8 * k + e];
  parts_of(y, p);
}
// Registers of the state: rows 32 t + 16 (r / 8) + 8 half + r % 8 of column c.
__device__ __forceinline__ int state_row(int t, int r) { return 32 * t + 16 * (r >> 3) + (r & 7); }

// The decays between a lane's token and the others of its window: g^|x - tok| for the 16 others x = 8 (r / 4) + 4 half + r % 4, of those up
// to it (ahead = false) or from it on; of its own half of the 32 only where two sequences share them.
template <bool PAIR>
__device__ __forceinline__ void decays(const float* pw, int tok, int half, bool ahead, float (&out)[16]) {
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const int x = 8 * (r >> 2) + 4 * half + (r & 3), d = ahead ? x - tok : tok - x;
    out[r] = d >= 0 && !(PAIR && (x ^ tok) & 16) ? pw[max(d, 0)] : 0.f;
  }
}
__device__ __forceinline__ void powers_of(float g, float* pw, int lane) {
  if (lane <= kTok) pw[lane] = power(g, lane);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
}

// 32 columns of the wave's 32 rows go out through LDS (`room`: 32 rows of kRoom units): a row's lanes then store it side by side, 16 bytes
// each, where the registers as they are would leave 16-byte pieces of 32 rows with each instruction, four times as many requests.
// base: the rows' first column; n0, n1: tokens of the first and, with PAIR, the second sequence.  Returns whether all were finite.
template <class T> constexpr int kRoom = 2 * (int)sizeof(T) + 1;
template <class T, bool PAIR>
__device__ __forceinline__ bool store_rows(T* base, int64_t st, int64_t sn, const floatx16& x, int width, int n0, int n1, bool wanted, uint4* room) {
  constexpr int PER = Elem<T>::kPer, UNITS = 32 / PER;
  const int lane = threadIdx.x & 63, half = lane >> 5, tok = lane & 31;
  float bad = 0.f;
#pragma unroll
  for (int r = 0; r < 16; ++r) bad = fmaf(x[r], 0.f, bad);
  T* mine = reinterpret_cast<T*>(room + tok * kRoom<T>) + 4 * half;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float y[4] = {x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
    store4(mine + 8 * q, y);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  const int u = lane % UNITS;
#pragma unroll
  for (int i = 0; i < 32 * UNITS / 64; ++i) {
    const int row = i * (64 / UNITS) + lane / UNITS, pos = PAIR ? row & 15 : row, slot = PAIR ? row >> 4 : 0;
    const uint4 v = room[row * kRoom<T> + u];
    if (wanted && u * PER < width && pos < (slot ? n1 : n0)) *reinterpret_cast<uint4*>(base + slot * sn + pos * st + u * PER) = v;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  return !__any(bad != 0.f);
}

// KD: dk rounded up to 16, 32, 64 or 128.  OUT: outputs are computed, else states alone.
// A wave goes over its rows' 32 tokens in turn and has the next ones' on the way while it works.  4 sequences of 8192, 8 heads of 64, bf16: 32 us
// for the states, 10 for the scan, 47 for the outputs; vector instructions (the parts of scores, keys and states) bound it at two waves a
// SIMD, whose 256 registers the outputs' kernel passes by 4, spilled.  In fp32 (211 us in all) a head of 64 takes one wave a SIMD; heads up to 16
// spill 4, up to 32 18, up to 128 6.  50 000 windows of 16, 8 heads of 16, states in and out: bf16 897 us, fp32 1184, half the wave's
// tokens idle and a window's states asked for when the one before has ended; 20 000 windows of 32, 4 heads of 32: 282 and 459 us.
template <class T, int KD, bool OUT>
__global__ __launch_bounds__(256, KD <= (sizeof(T) == 2 ? 64 : 32) ? 2 : 1) void k_decay(DecayArgs a) {
  constexpr int KC = KD / 16, KT = (KD + 31) / 32, IN = Kind<T>::kIn, MID = Kind<T>::kMid;
  __shared__ float pw_lds[4][kTok + 4];
  __shared__ uint4 room_lds[OUT ? 4 : 1][32 * kRoom<T>];
  const int lane = threadIdx.x & 63, half = lane >> 5, tok = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float* pw = pw_lds[wave];
  // a wave keeps to one head and block of columns and takes sequences (of a segment) that lie side by side
  const uint32_t line = blockIdx.x * 4 + wave, across = (uint32_t)(a.heads * a.blocks_v), rows = (uint32_t)(a.N * a.segs);
  const int h = line % across / a.blocks_v, b = line % a.blocks_v;
  uint32_t row = line / across * a.run;
  const uint32_t row_end = min(rows, row + a.run);
  if (row >= rows) return;
  const float g = a.decay[h];
  powers_of(g, pw, lane);
  float near[16];                                                // g^(i-j) of the lane's scores
  decays<false>(pw, tok, half, false, near);
  const float fade0 = pw[tok], fade1 = pw[tok + 1];              // g^i, g^(i+1)

  struct Item {
    int seg;
    int64_t i, n, p0, p_hi;
  };
  auto begin = [&](uint32_t row) {
    Item it;
    it.i = row % (uint32_t)a.N;
    it.seg = row / (uint32_t)a.N;
    it.n = a.T;
    if (a.lengths) it.n = __builtin_amdgcn_readfirstlane(min((int)min(a.T, (int64_t)INT32_MAX), max(a.lengths[it.i], 0)));
    it.p0 = it.seg * a.seg_len;
    it.p_hi = min(it.n, it.p0 + a.seg_len);
    return it;
  };
  auto from = [&](const Rows& x, int width, const Item& it) {    // the item's first row, and from one token's row to the next
    const int64_t t = a.reversed ? it.n - 1 - it.p0 : it.p0;
    return static_cast<const T*>(x.p) + t * x.st + it.i * x.sn + (int64_t)h * width;
  };
  const int64_t way = a.reversed ? -1 : 1;
  const int64_t offA = way * tok * a.A.st + 8 * half, offB = way * tok * a.B.st + 8 * half, offC = way * tok * a.C.st + 8 * half;
  Raw8<T> rawA[KC], rawB[KC], rawC[2];
  bool flag = false;
  auto fetch = [&](const Item& it) {
    const bool on = tok < it.p_hi - it.p0;
    const T* pb = from(a.B, a.dk, it) + offB;
    const T* pc = from(a.C, a.dv, it) + 32 * b + offC;
#pragma unroll
    for (int k = 0; k < 2; ++k) rawC[k] = fetch8(pc + 16 * k, on && 32 * b + 16 * k + 8 * half < a.dv);
#pragma unroll
    for (int k = 0; k < KC; ++k) rawB[k] = fetch8(pb + 16 * k, on && 16 * k + 8 * half < a.dk);
    if constexpr (OUT) {
      const T* pa = from(a.A, a.dk, it) + offA;
#pragma unroll
      for (int k = 0; k < KC; ++k) rawA[k] = fetch8(pa + 16 * k, on && 16 * k + 8 * half < a.dk);
    }
    flag = false;
    if (a.reset && on && half == 0) {
      const int64_t pos = it.p0 + tok;
      if (!a.reversed) flag = a.reset[pos * a.N + it.i] != 0;
      else if (pos > 0) flag = a.reset[(it.n - pos) * a.N + it.i] != 0;
    }
  };

  Item it = begin(row);
  fetch(it);
  floatx16 S[KT];
  bool holds = false, cut = false, fresh_unit = true;    // holds: the state may be other than zero; cut: a reset was met
  while (true) {
    const int dv0 = 32 * b, c = dv0 + tok;            // c: the lane's column of the state
    const int64_t state_at = (((int64_t)it.seg * a.N + it.i) * a.heads + h) * a.dk * a.dv;
    if (fresh_unit) {
      const float* in = a.s_in + state_at + 8 * half * a.in_r + c * a.in_c;
#pragma unroll
      for (int t = 0; t < KT; ++t) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          S[t][r] = a.s_in && state_row(t, r) + 8 * half < a.dk && c < a.dv ? in[state_row(t, r) * a.in_r] : 0.f;
      }
      holds = a.s_in != nullptr;
      cut = false;
    }
    const int64_t p0 = it.p0, n = it.n;
    const int m = (int)min((int64_t)kTok, it.p_hi - p0);      // may be none
    const bool fresh = a.reversed && p0 == 0;     // the state that comes in is that of the first token, not of one before
    const bool unit_ends = p0 + kTok >= it.p_hi;
    const bool step = !OUT || a.s_out || !unit_ends;          // whether the state is wanted after these tokens
    uint32_t resets = 0;
    if (a.reset) {
      resets = (uint32_t)__ballot(flag);
      cut |= resets != 0;
    }
    floatx16 P = {}, inter = {}, Bc[KT], Cc = {};
#pragma unroll
    for (int t = 0; t < KT; ++t) Bc[t] = floatx16{};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (dv0 + 16 * k < a.dv) {
        uint4 f[IN];
        operand(rawC[k], f);
        mul(Cc, f, {identity(k, half, tok)});
      }
    }
#pragma unroll
    for (int k = 0; k < KC; ++k) {
      uint4 fb[IN];
      operand(rawB[k], fb);
      if constexpr (OUT) {
        uint4 fa[IN];
        operand(rawA[k], fa);
        mul(P, fb, fa);
        if (holds) {
          uint4 fs[MID];
          half_parts(S[k / 2], k & 1, fs);
          mul(inter, fs, fa);
        }
      }
      if (step) mul(Bc[k / 2], fb, {identity(k & 1, half, swap23(tok))});
    }
    // the next rows, on their way from here on
    Item next = it;
    next.p0 += kTok;
    if (unit_ends) ++row;
    const bool more = !unit_ends || row < row_end;
    if (unit_ends && more) next = begin(row);
    if (more) fetch(next);

    uint4 fc[2][IN];      // C with its tokens as the contraction
#pragma unroll
    for (int k = 0; k < 2; ++k) half_parts(Cc, k, fc[k]);
    float bad = 0.f;
    if constexpr (OUT) {
      const uint32_t before = resets & ((2u << tok) - 1u);       // resets up to the lane's token (2 << 31 is 0: all of them)
      floatx16 intra = {};
#pragma unroll
      for (int r = 0; r < 16; ++r) P[r] *= near[r];    // a score that is not finite leaves an output that is not
      if (resets) {
        const int since = before ? 31 - __clz(before) : 0;
#pragma unroll
        for (int r = 0; r < 16; ++r) P[r] = 8 * (r >> 2) + 4 * half + (r & 3) >= since ? P[r] : 0.f;
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (16 * k < m) {
          uint4 fp[MID];
          half_parts(P, k, fp);
          mul(intra, fc[k], fp);
        }
      }
      const float f = a.gam * (fresh ? fade0 : fade1);
      const bool sees = holds && !before;
#pragma unroll
      for (int r = 0; r < 16; ++r) P[r] = fmaf(a.alpha, intra[r], sees ? f * inter[r] : 0.f);
      bad = store_rows<T, false>(const_cast<T*>(from(a.O, a.dv, it)) + dv0, way * a.O.st, 0, P, a.dv - dv0, m, 0, true, room_lds[wave]) ? 0.f : 1.f;
    } else {
      not_finite(bad, Cc);
#pragma unroll
      for (int t = 0; t < KT; ++t) { not_finite(bad, Bc[t]); not_finite(bad, S[t]); }
    }
    if (__builtin_expect(__any(bad != 0.f), 0)) {
      __threadfence();      // other lanes wrote these rows above
      // One by one, over what was stored: the state for each token, its row's product with it.  (An output is not finite
      // wherever a value among the tokens or in the state is not.)
      for (int q = 0; q < m; ++q) {
        const int64_t at = a.reversed ? n - 1 - (p0 + q) : p0 + q;
        const T* qa = static_cast<const T*>(a.A.p) + at * a.A.st + it.i * a.A.sn + (int64_t)h * a.dk + 8 * half;
        const T* qb = static_cast<const T*>(a.B.p) + at * a.B.st + it.i * a.B.sn + (int64_t)h * a.dk + 8 * half;
        const float vc = c < a.dv ? to_float((static_cast<const T*>(a.C.p) + at * a.C.st + it.i * a.C.sn + (int64_t)h * a.dv)[c]) : 0.f;
        const bool zero = resets >> q & 1;
        const float keep = fresh && q == 0 ? 1.f : g;
        float o = 0.f;
#pragma unroll
        for (int t = 0; t < KT; ++t) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            if (state_row(t, r) + 8 * half < a.dk && c < a.dv) {
              const float old = zero ? 0.f : holds || q > 0 ? keep * S[t][r] : 0.f;
              S[t][r] = fmaf(a.beta * to_float(qb[state_row(t, r)]), vc, old);
              if constexpr (OUT) o = fmaf(to_float(qa[state_row(t, r)]), S[t][r], o);
            }
          }
        }
        if constexpr (OUT) {
          o += __shfl_xor(o, 32);
          if (half == 0 && c < a.dv)
            (static_cast<T*>(const_cast<void*>(a.O.p)) + at * a.O.st + it.i * a.O.sn + (int64_t)h * a.dv)[c] = Elem<T>::one(a.gam * o);
        }
      }
      holds |= m > 0;
    } else if (step && m > 0) {
      const int last = resets ? 31 - __clz(resets) : 0;
      const float keep = resets ? 0.f : pw[m - (fresh ? 1 : 0)];
      float w[16];
      if (m == kTok && !resets) {
#pragma unroll
        for (int r = 0; r < 16; ++r) w[r] = a.beta * pw[kTok - 1 - (8 * (r >> 2) + 4 * half + (r & 3))];
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int j = 8 * (r >> 2) + 4 * half + (r & 3);
          w[r] = j < m && j >= last ? a.beta * pw[max(m - 1 - j, 0)] : 0.f;
        }
      }
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        floatx16 U = {};
#pragma unroll
        for (int r = 0; r < 16; ++r) Bc[t][r] *= w[r];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          if (16 * k < m) {
            uint4 fb[3];
            half_parts(Bc[t], k, fb);
            mul(U, fb, fc[k]);
          }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) S[t][r] = fmaf(resets ? 0.f : S[t][r], keep, U[r]);   // what a reset drops may be infinite
      }
      holds = true;
    }
    if (unit_ends) {
      if (a.s_out) {
        float f = 1.f;
        const bool drop = a.out_link && n > 0 && a.reset && a.reset[it.i];
        if (a.out_link && n > 0) f = g;
        float* out = a.s_out + state_at + 8 * half * a.out_r + c * a.out_c;
#pragma unroll
        for (int t = 0; t < KT; ++t) {
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            if (state_row(t, r) + 8 * half < a.dk && c < a.dv) out[state_row(t, r) * a.out_r] = drop ? 0.f : f * S[t][r];
          }
        }
      }
      if (!OUT && a.factor && b == 0 && lane == 0) {
        const int64_t len = max(it.p_hi - it.seg * a.seg_len, (int64_t)0);
        a.factor[((int64_t)it.seg * a.N + it.i) * a.heads + h] = cut ? -1.f : power(g, (uint32_t)(len - (a.reversed && it.seg == 0 && len > 0 ? 1 : 0)));
      }
    }
    if (!more) return;
    fresh_unit = unit_ends;
    it = next;
  }
}

// ---------------------------------------------------------------------------------------------- windows of up to 32 tokens

// A window's outputs one row of the state after the other: what is done where a value is not finite.  acc: [32][64] floats of the wave.
template <class T>
struct Walk {
  const T* A; const T* B; const T* C; T* O;     // the sequence's and head's first rows
  int64_t sa, sb, sc, so;                       // from token to token
  int n, da, dc;
  bool reversed;
  float g, beta, gam;
  const uint8_t* reset; int64_t reset_st;       // the sequence's first flag
  const float* in; int in_r, in_c;
  float* out;                                   // [da][dc]: the last state times l_0 g
};
template <class T>
__device__ void walk_window(const Walk<T>& w, float* acc) {
  const int lane = threadIdx.x & 63, half = lane >> 5;
  for (int b = 0; b < w.dc; b += 32) {
    const int c = b + (lane & 31);
    const bool have = c < w.dc;
    for (int p = 0; p < w.n; ++p) acc[p * 64 + lane] = 0.f;
    for (int r = half; r < w.da; r += 2) {
      float s = w.in && have ? w.in[r * w.in_r + c * w.in_c] : 0.f;
      for (int p = 0; p < w.n; ++p) {
        const int64_t t = w.reversed ? w.n - 1 - p : p;
        if (p > 0 || !w.reversed) {
          const bool cut = w.reset && w.reset[(w.reversed ? t + 1 : t) * w.reset_st];
          s = cut || (p == 0 && !w.in) ? 0.f : w.g * s;
        }
        if (have) {
          s = fmaf(w.beta * to_float(w.B[t * w.sb + r]), to_float(w.C[t * w.sc + c]), s);
          acc[p * 64 + lane] = fmaf(to_float(w.A[t * w.sa + r]), s, acc[p * 64 + lane]);
        }
      }
      if (w.out && have) w.out[r * w.dc + c] = w.n == 0 ? s : w.reset && w.reset[0] ? 0.f : w.g * s;
    }
    if (!w.O) continue;
    for (int p = 0; p < w.n; ++p) {
      const float o = acc[p * 64 + lane] + __shfl_xor(acc[p * 64 + lane], 32);
      const int64_t t = w.reversed ? w.n - 1 - p : p;
      if (have && half == 0) w.O[t * w.so + c] = Elem<T>::one(w.gam * o);
    }
  }
}

// The forward pass of windows of up to 32 tokens from zero states, the states not wanted: nothing is carried.  Two sequences
// of up to 16 tokens share the 32 of a wave (PAIR).  100 000 windows of 16, 8 heads of 16: 365 us, 4.5 TB/s; memory bounds it (fp32, 50 000: 404).
template <class T, int KD, bool PAIR>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? (KD <= 32 ? 3 : 2) : (KD <= 64 ? 2 : 1)) void k_decay_window(DecayArgs a) {
  constexpr int KC = KD / 16, IN = Kind<T>::kIn, MID = Kind<T>::kMid, PER = PAIR ? 2 : 1;
  __shared__ float pw_lds[4][kTok + 4];
  __shared__ __align__(16) float walk_lds[4][32 * 64];
  const int lane = threadIdx.x & 63, half = lane >> 5, tok = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int slot = PAIR ? tok >> 4 : 0, pos = PAIR ? tok & 15 : tok;
  float* pw = pw_lds[wave];
  const uint32_t line = blockIdx.x * 4 + wave, across = (uint32_t)(a.heads * a.blocks_v), rows = (uint32_t)((a.N + PER - 1) / PER);
  const int h = line % across / a.blocks_v, dv0 = 32 * (line % a.blocks_v);
  uint32_t row = line / across * a.run;
  const uint32_t row_end = min(rows, row + a.run);
  if (row >= rows) return;
  // Narrow heads share cache lines with their neighbours, which the workgroup's other waves read: where all four take the same rows
  // they fetch in step, and each line comes into the L1 cache once (100 000 windows of 16, 8 heads of 16: 451 us apart, 410 in step, when the
  // outputs left the registers as they were).
  const bool together = (across & 3) == 0;
  const int64_t offA = slot * a.A.sn + pos * a.A.st + 8 * half, offB = slot * a.B.sn + pos * a.B.st + 8 * half;
  const int64_t offC = slot * a.C.sn + pos * a.C.st + 8 * half;
  const float g = a.decay[h];
  powers_of(g, pw, lane);
  float near[16];
  decays<PAIR>(pw, tok, half, false, near);
  auto tokens = [&](uint32_t row) {      // of the lane's sequence
    const int64_t i = (int64_t)row * PER + slot;
    if (i >= a.N) return 0;
    return a.lengths ? min((int)a.T, max(a.lengths[i], 0)) : (int)a.T;
  };
  Raw8<T> rawA[KC], rawB[KC], rawC[2];
  bool flag = false;
  auto fetch = [&](uint32_t row, int n) {
    const bool on = pos < n;
    const int64_t i = (int64_t)row * PER;
    const T* pa = static_cast<const T*>(a.A.p) + i * a.A.sn + (int64_t)h * a.dk + offA;
    const T* pb = static_cast<const T*>(a.B.p) + i * a.B.sn + (int64_t)h * a.dk + offB;
    const T* pc = static_cast<const T*>(a.C.p) + i * a.C.sn + (int64_t)h * a.dv + dv0 + offC;
#pragma unroll
    for (int k = 0; k < KC; ++k) {
      rawB[k] = fetch8(pb + 16 * k, on && 16 * k + 8 * half < a.dk);
      rawA[k] = fetch8(pa + 16 * k, on && 16 * k + 8 * half < a.dk);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) rawC[k] = fetch8(pc + 16 * k, on && dv0 + 16 * k + 8 * half < a.dv);
    flag = a.reset && on && half == 0 && a.reset[pos * a.N + i + slot] != 0;
  };

  int n_next = tokens(row);
  int n = n_next;
  fetch(row, n);
  n_next = row + 1 < row_end ? tokens(row + 1) : 0;
  while (true) {
    const int64_t i0 = (int64_t)row * PER;
    const uint32_t resets = a.reset ? (uint32_t)__ballot(flag) : 0;
    floatx16 P = {}, Cc = {}, out = {};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (dv0 + 16 * k < a.dv) {
        uint4 f[IN];
        operand(rawC[k], f);
        mul(Cc, f, {identity(k, half, tok)});
      }
    }
#pragma unroll
    for (int k = 0; k < KC; ++k) {
      uint4 fa[IN], fb[IN];
      operand(rawA[k], fa);
      operand(rawB[k], fb);
      mul(P, fb, fa);
    }
    const int n_this = n;
    if (together) __builtin_amdgcn_s_barrier();
    if (++row < row_end) {
      fetch(row, n_next);
      n = n_next;
      n_next = row + 1 < row_end ? tokens(row + 1) : 0;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) P[r] *= near[r];    // a score that is not finite leaves an output that is not
    if (resets) {
      const uint32_t before = resets & ((2u << tok) - 1u) & (PAIR ? 0xffffu << (16 * slot) : ~0u);
      const int since = before ? 31 - __clz(before) : 0;
#pragma unroll
      for (int r = 0; r < 16; ++r) P[r] = 8 * (r >> 2) + 4 * half + (r & 3) >= since ? P[r] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      uint4 fc[IN], fp[MID];
      half_parts(Cc, k, fc);
      half_parts(P, k, fp);
      mul(out, fc, fp);
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) out[r] *= a.alpha;
    T* O = static_cast<T*>(const_cast<void*>(a.O.p));
    const int64_t at = i0 * a.O.sn + (int64_t)h * a.dv;
    const int n0 = __builtin_amdgcn_readfirstlane(n_this), n1 = PAIR ? __builtin_amdgcn_readlane(n_this, 16) : 0;
    if (__builtin_expect(!store_rows<T, PAIR>(O + at + dv0, a.O.st, a.O.sn, out, a.dv - dv0, n0, n1, true, reinterpret_cast<uint4*>(walk_lds[wave])), 0)) {
      __threadfence();      // other lanes wrote these rows above
      for (int q = 0; q < PER; ++q) {
        const int64_t i = i0 + q;
        const int live = q ? n1 : n0;
        const T *A = static_cast<const T*>(a.A.p), *B = static_cast<const T*>(a.B.p), *C = static_cast<const T*>(a.C.p);
        const Walk<T> w{A + i * a.A.sn + h * a.dk, B + i * a.B.sn + h * a.dk, C + i * a.C.sn + h * a.dv + dv0, O + i * a.O.sn + h * a.dv + dv0,
                        a.A.st, a.B.st, a.C.st, a.O.st, live, a.dk, min(32, a.dv - dv0), false, g, a.beta, a.gam,
                        a.reset ? a.reset + i : nullptr, a.N, nullptr, 0, 0, nullptr};
        if (live > 0) walk_window(w, walk_lds[wave]);
      }
    }
    if (row >= row_end) return;
  }
}

struct BackArgs {
  Rows q, k, v, go, dq, dkey, dval;
  int64_t T, N;
  int32_t heads, dk, dv;
  const float* decay;
  float scale;
  const float* s0;
  const float* dsn;
  float* ds0;
  const int32_t* lengths;
  const uint8_t* reset;
  uint32_t run;
};

// All gradients of windows of up to 32 tokens, every tensor read once: dk, dv up to KD.  States (not with PAIR) are read and written as
// they are needed: nothing is carried.  20 000 ragged windows of 32, 4 heads of 32, with states: 457 us, 3.4 TB/s; the registers (256, and
// nine spilled) leave two waves a SIMD, which do not cover all waits.  In fp32 that takes 1338 us at one wave a SIMD; fp32 heads up to 16 with states
// spill 60 registers, up to 64 134 (4000 windows of 16, 8 heads of 64: 2863 us, bf16 1276).  (Three passes of k_decay took 900.)
template <class T, int KD, bool PAIR>
__global__ __launch_bounds__(256, KD <= (sizeof(T) == 2 ? 32 : 16) ? 2 : 1) void k_decay_window_back(BackArgs a) {
  constexpr int KC = KD / 16, KT = (KD + 31) / 32, IN = Kind<T>::kIn, MID = Kind<T>::kMid, PER = PAIR ? 2 : 1;
  __shared__ float pw_lds[4][kTok + 4];
  __shared__ __align__(16) float walk_lds[4][32 * 64];
  __shared__ uint4 room_lds[4][32 * kRoom<T>];
  const int lane = threadIdx.x & 63, half = lane >> 5, tok = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int slot = PAIR ? tok >> 4 : 0, pos = PAIR ? tok & 15 : tok;
  float* pw = pw_lds[wave];
  const uint32_t line = blockIdx.x * 4 + wave, rows = (uint32_t)((a.N + PER - 1) / PER);
  const int h = line % a.heads;
  uint32_t row = line / a.heads * a.run;
  const uint32_t row_end = min(rows, row + a.run);
  if (row >= rows) return;
  const float g = a.decay[h];
  powers_of(g, pw, lane);
  // [32 rows][8 units] each; what the walk sums in takes the same place
  uint4 *s0_lds = reinterpret_cast<uint4*>(walk_lds[wave]), *dsn_lds = s0_lds + 256;
  const int part_row = lane / 8, part_unit = lane % 8, part_at = 8 * part_row + (part_unit ^ part_row);    // the lane's unit of 8 rows
  auto tokens = [&](uint32_t row) {
    const int64_t i = (int64_t)row * PER + slot;
    if (i >= a.N) return 0;
    return a.lengths ? min((int)a.T, max(a.lengths[i], 0)) : (int)a.T;
  };
  auto place = [&](const Rows& x, int width, uint32_t row) {   // the lane's row
    return static_cast<const T*>(x.p) + ((int64_t)row * PER + slot) * x.sn + pos * x.st + (int64_t)h * width;
  };
  Raw8<T> rawq[KC], rawk[KC], rawv[KC], rawd[KC];
  bool flag = false;
  auto fetch = [&](uint32_t row, int n) {
    const bool on = pos < n;
    const T *pq = place(a.q, a.dk, row) + 8 * half, *pk = place(a.k, a.dk, row) + 8 * half;
    const T *pv = place(a.v, a.dv, row) + 8 * half, *pd = place(a.go, a.dv, row) + 8 * half;
#pragma unroll
    for (int k = 0; k < KC; ++k) {
      const bool ink = on && 16 * k + 8 * half < a.dk, inv = on && 16 * k + 8 * half < a.dv;
      rawq[k] = fetch8(pq + 16 * k, ink);
      rawk[k] = fetch8(pk + 16 * k, ink);
      rawv[k] = fetch8(pv + 16 * k, inv);
      rawd[k] = fetch8(pd + 16 * k, inv);
    }
    flag = a.reset && on && half == 0 && a.reset[pos * a.N + (int64_t)row * PER + slot] != 0;
  };

  int n = tokens(row), n_next = row + 1 < row_end ? tokens(row + 1) : 0;
  fetch(row, n);
  while (true) {
    const int64_t i0 = (int64_t)row * PER, state = (i0 * a.heads + h) * a.dk * a.dv;
    const uint32_t resets = a.reset ? (uint32_t)__ballot(flag) : 0;
    const uint32_t own = PAIR ? 0xffffu << (16 * slot) : ~0u;
    const uint32_t before = resets & ((2u << tok) - 1u) & own, after = resets & ~((2u << tok) - 1u) & own;
    const float *s0 = a.s0 + state, *dsn = a.dsn + state;
    // eight numbers of a state for the lane's output column: along row r of it, or down column c
    auto along = [&](const float* s, int r, int c, float (&x)[8]) {
      const bool in = s && r < a.dk && c < a.dv;
      const float4 none = make_float4(0.f, 0.f, 0.f, 0.f), *at = reinterpret_cast<const float4*>(s + r * a.dv + c);
      const float4 lo = in ? at[0] : none, hi = in ? at[1] : none;
      x[0] = lo.x; x[1] = lo.y; x[2] = lo.z; x[3] = lo.w; x[4] = hi.x; x[5] = hi.y; x[6] = hi.z; x[7] = hi.w;
    };
    auto down = [&](const float* s, int r, int c, float (&x)[8]) {
      const bool in = s && r < a.dk && c < a.dv;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = in ? s[(r + e) * a.dv + c] : 0.f;
    };
    // States of up to 32 x 32 go through LDS, on their way there while the first scores are worked out: their rows and columns are then
    // at hand for all that reads them.  A 16-byte unit's place in its row is turned by the row, so that neither way meets in a bank.
    constexpr bool STAGED = !PAIR && KT == 1;
    Raw8<uint16_t> s0_raw[4], dsn_raw[4];
    if constexpr (STAGED) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 8 * i + part_row;
        const bool in = r < a.dk && 4 * part_unit < a.dv;      // zeros behind a narrower state
        s0_raw[i] = fetch8(reinterpret_cast<const uint16_t*>(s0 + r * a.dv + 4 * part_unit), a.s0 && in);
        dsn_raw[i] = fetch8(reinterpret_cast<const uint16_t*>(dsn + r * a.dv + 4 * part_unit), a.dsn && in);
      }
    }
    auto staged_row = [&](const uint4* s, int r, int c, float (&x)[8]) {
      Elem<float>::unpack(s[r * 8 + (c / 4 ^ (r & 7))], x);
      Elem<float>::unpack(s[r * 8 + ((c / 4 + 1) ^ (r & 7))], x + 4);
    };
    auto staged_col = [&](const uint4* s, int r, int c, float (&x)[8]) {
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = reinterpret_cast<const float*>(s)[((r + e) * 8 + (c / 4 ^ ((r + e) & 7))) * 4 + (c & 3)];
    };
    uint4 fq[KC][IN], fk[KC][IN], fv[KC][IN], fd[KC][IN];
#pragma unroll
    for (int k = 0; k < KC; ++k) {
      operand(rawq[k], fq[k]);
      operand(rawk[k], fk[k]);
      operand(rawv[k], fv[k]);
      operand(rawd[k], fd[k]);
    }
    const int n_this = n;
    if (++row < row_end) {
      fetch(row, n_next);
      n = n_next;
      n_next = row + 1 < row_end ? tokens(row + 1) : 0;
    }
    // the lane's token as the one that reads (the others before it) or that is read (from it on), with what lies between
    auto scores = [&](const uint4 (&f)[KC][IN], const uint4 (&own)[KC][IN], bool ahead, uint4 (&score)[2][MID]) {
      floatx16 x = {};
#pragma unroll
      for (int k = 0; k < KC; ++k) mul(x, f[k], own[k]);
      float w[16];
      decays<PAIR>(pw, tok, half, ahead, w);
      const int since = before ? 31 - __clz(before) : 0, until = after ? __ffs(after) - 1 : 32;
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] *= w[r];
      if (resets) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int o = 8 * (r >> 2) + 4 * half + (r & 3);
          x[r] = (ahead ? o < until : o >= since) ? x[r] : 0.f;
        }
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) half_parts(x, k, score[k]);
    };
    // a tensor's 32 columns with its tokens as the contraction
    auto columns = [&](const uint4 (&f)[KC][IN], int t, floatx16& x, int order) {
      x = floatx16{};
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        if (2 * t + k < KC) mul(x, f[2 * t + k < KC ? 2 * t + k : 0], {identity(k, half, order)});
      }
    };
    auto sums = [&](const floatx16& x, const uint4 (&score)[2][MID], floatx16& out) {
      out = floatx16{};
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        uint4 f[IN];
        half_parts(x, k, f);
        mul(out, f, score[k]);
      }
    };
    const int live0 = __builtin_amdgcn_readfirstlane(n_this), live1 = PAIR ? __builtin_amdgcn_readlane(n_this, 16) : 0;
    const int n0 = PAIR ? 0 : live0;
    const int last = resets ? 31 - __clz(resets) : 0;
    const bool lasts = tok < n0 && tok >= last;                  // whether the last state holds something of the lane's token
    const float fade = a.scale * pw[tok + 1], keep = pw[max(n0 - 1 - tok, 0)];   // S0 in the token, the token in the last state
    bool fine = true;
    auto leave = [&](const Rows& out, int width, int t, const floatx16& sum, const floatx16& far, bool sees, float weight) {
      floatx16 x;
#pragma unroll
      for (int r = 0; r < 16; ++r) x[r] = a.scale * sum[r] + (!PAIR && sees ? weight * far[r] : 0.f);
      T* base = static_cast<T*>(const_cast<void*>(out.p)) + i0 * out.sn + (int64_t)h * width + 32 * t;
      fine &= store_rows<T, PAIR>(base, out.st, out.sn, x, width - 32 * t, live0, live1, out.p != nullptr, room_lds[wave]);
    };
    {   // dq
      uint4 score[2][MID];
      scores(fv, fd, false, score);
      if constexpr (STAGED) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s0_lds[64 * i + part_at] = s0_raw[i].w[0];
          dsn_lds[64 * i + part_at] = dsn_raw[i].w[0];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      }
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        if (32 * t >= a.dk) break;
        floatx16 x, out, far = {};
        columns(fk, t, x, tok);
        sums(x, score, out);
        if (!PAIR && a.s0) {
#pragma unroll
          for (int k = 0; k < KC; ++k) {
            uint4 f[MID];
            if constexpr (STAGED) {
              float y[8];
              staged_row(s0_lds, tok, 16 * k + 8 * half, y);
              parts_of(y, f);
            } else {
              float y[8];
              along(s0, 32 * t + tok, 16 * k + 8 * half, y);
              parts_of(y, f);
            }
            mul(far, f, fd[k]);
          }
        }
        leave(a.dq, a.dk, t, out, far, a.s0 && !before, fade);
      }
    }
    __builtin_amdgcn_sched_barrier(0);      // one gradient's scores and sums at a time: all three at once do not fit the registers
    {   // dk
      uint4 score[2][MID];
      scores(fd, fv, true, score);
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        if (32 * t >= a.dk) break;
        floatx16 x, out, far = {};
        columns(fq, t, x, tok);
        sums(x, score, out);
        if (!PAIR && a.dsn) {
#pragma unroll
          for (int k = 0; k < KC; ++k) {
            uint4 f[MID];
            if constexpr (STAGED) {
              float y[8];
              staged_row(dsn_lds, tok, 16 * k + 8 * half, y);
              parts_of(y, f);
            } else {
              float y[8];
              along(dsn, 32 * t + tok, 16 * k + 8 * half, y);
              parts_of(y, f);
            }
            mul(far, f, fv[k]);
          }
        }
        leave(a.dkey, a.dk, t, out, far, a.dsn && lasts, keep);
      }
    }
    __builtin_amdgcn_sched_barrier(0);      // one gradient's scores and sums at a time: all three at once do not fit the registers
    {   // dv
      uint4 score[2][MID];
      scores(fq, fk, true, score);
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        if (32 * t >= a.dv) break;
        floatx16 x, out, far = {};
        columns(fd, t, x, tok);
        sums(x, score, out);
        if (!PAIR && a.dsn) {
#pragma unroll
          for (int k = 0; k < KC; ++k) {
            uint4 f[MID];
            if constexpr (STAGED) {
              float y[8];
              staged_col(dsn_lds, 16 * k + 8 * half, tok, y);
              parts_of(y, f);
            } else {
              float y[8];
              down(dsn, 16 * k + 8 * half, 32 * t + tok, y);
              parts_of(y, f);
            }
            mul(far, f, fk[k]);
          }
        }
        leave(a.dval, a.dv, t, out, far, a.dsn && lasts, keep);
      }
    }
    __builtin_amdgcn_sched_barrier(0);      // one gradient's scores and sums at a time: all three at once do not fit the registers
    if (__builtin_expect(!fine, 0)) {
      __threadfence();      // other lanes wrote these rows above
      for (int q = 0; q < PER; ++q) {
        const int64_t i = i0 + q;
        const int live = q ? live1 : live0;
        auto at = [&](const Rows& x, int width) { return x.p ? static_cast<T*>(const_cast<void*>(x.p)) + i * x.sn + (int64_t)h * width : nullptr; };
        const uint8_t* reset = a.reset ? a.reset + i : nullptr;
        const int m = a.dk, c = a.dv;
        if (PAIR && live == 0) continue;
        walk_window(Walk<T>{at(a.go, c), at(a.v, c), at(a.k, m), at(a.dq, m), a.go.st, a.v.st, a.k.st, a.dq.st, live, c, m, false, g, 1.f, a.scale, reset, a.N,
                            !PAIR && a.s0 ? s0 : nullptr, 1, c, nullptr}, walk_lds[wave]);
        walk_window(Walk<T>{at(a.v, c), at(a.go, c), at(a.q, m), at(a.dkey, m), a.v.st, a.go.st, a.q.st, a.dkey.st, live, c, m, true, g, a.scale, 1.f, reset, a.N,
                            !PAIR && a.dsn ? dsn : nullptr, 1, c, nullptr}, walk_lds[wave]);
        walk_window(Walk<T>{at(a.k, m), at(a.q, m), at(a.go, c), at(a.dval, c), a.k.st, a.q.st, a.go.st, a.dval.st, live, m, c, true, g, a.scale, 1.f, reset, a.N,
                            !PAIR && a.dsn ? dsn : nullptr, c, 1, !PAIR && a.ds0 ? a.ds0 + state : nullptr}, walk_lds[wave]);
      }
    } else if (!PAIR && a.ds0) {      // after all that reads dsn, which may be in its place
      const int until = resets ? __ffs(resets) - 1 : 32;        // the tokens that S0 reaches are those before it
      const float pass = pw[n0];
#pragma unroll
      for (int t = 0; t < KT; ++t) {
        if (32 * t >= a.dv) break;
        floatx16 x;
        columns(fd, t, x, tok);
        uint4 fx[2][IN];
#pragma unroll
        for (int k = 0; k < 2; ++k) half_parts(x, k, fx[k]);
#pragma unroll
        for (int u = 0; u < KT; ++u) {
          if (32 * u >= a.dk) break;
          floatx16 y, S = {};
          columns(fq, u, y, swap23(tok));     // dS0's rows in the order of `down`
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int o = 8 * (r >> 2) + 4 * half + (r & 3);
            y[r] = o < until ? y[r] * (a.scale * pw[o + 1]) : 0.f;
          }
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            uint4 f[3];
            half_parts(y, k, f);
            mul(S, f, fx[k]);
          }
          const int c = 32 * t + tok;
          float* to = a.ds0 + state + (int64_t)(32 * u + 8 * half) * a.dv + c;
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float in[8];
            if constexpr (STAGED) staged_col(dsn_lds, 16 * k + 8 * half, tok, in);
            else down(a.dsn ? dsn : nullptr, 32 * u + 16 * k + 8 * half, c, in);
            if (32 * u + 16 * k + 8 * half < a.dk && c < a.dv) {
#pragma unroll
              for (int e = 0; e < 8; ++e) to[(16 * k + e) * a.dv] = a.dsn && !resets ? fmaf(pass, in[e], S[8 * k + e]) : S[8 * k + e];
            }
          }
        }
      }
    }
    if (row >= row_end) return;
  }
}

// Joins the segments' own states: in place, each becomes the state that enters its segment; the last one goes to s_out.
struct ScanArgs {
  float* states;            // [segs][N][heads][dk dv]
  const float* factor;
  const float* s_in;        // [N][heads][dk dv] or nullptr
  float* s_out;             // the same, or nullptr
  int64_t N;
  int32_t heads, size, segs;
  int32_t out_link;
  const float* decay;
  const uint8_t* reset;
  const int32_t* lengths;
};
__global__ __launch_bounds__(256) void k_decay_scan(ScanArgs a) {
  const int64_t seqs = a.N * a.heads, all = seqs * a.size;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < all; e += (int64_t)gridDim.x * 256) {
    const int64_t ih = e / a.size;
    const float g = a.decay[ih % a.heads];
    float s = a.s_in ? a.s_in[e] : 0.f;
    for (int base = 0; base < a.segs; base += 8) {       // eight on their way at a time
      float own[8], f[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const bool in = base + k < a.segs;
        f[k] = in ? a.factor[(base + k) * seqs + ih] : 1.f;
        own[k] = in ? a.states[(base + k) * all + e] : 0.f;
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (base + k < a.segs) {
          a.states[(base + k) * all + e] = s;
          // a power that is zero only in fp32 leaves an infinity what it is
          if (f[k] == 0.f && g != 0.f) s = fabsf(s) <= 3.4028235e38f ? own[k] : s + own[k];
          else s = f[k] < 0.f ? own[k] : fmaf(f[k], s, own[k]);
        }
      }
    }
    if (a.s_out) {
      const int64_t i = ih / a.heads;
      if (a.out_link && (!a.lengths || a.lengths[i] > 0)) s = a.reset && a.reset[i] ? 0.f : g * s;
      a.s_out[e] = s;
    }
  }
}

// One token (4000 of them over 8 fp32 states of 64 x 64: 197 us, 5.3 TB/s): a wave a sequence and head, dv / 4 lanes a row of the state, as many rows at a time as fit, eight times.
template <class T>
__global__ __launch_bounds__(256) void k_decay_step(DecayArgs a) {
  __shared__ float4 sums[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int lv = a.dv / 4, rows = 64 / lv, sub = lane / lv, col = lane % lv * 4;
  const bool on = sub < rows;
  constexpr int U = 8;
  const int64_t units = a.N * a.heads;
  for (int64_t unit = (int64_t)blockIdx.x * 4 + wave; unit < units; unit += (int64_t)gridDim.x * 4) {
    const int64_t i = unit / a.heads;
    const int h = (int)(unit % a.heads);
    const bool live = !a.lengths || a.lengths[i] > 0;
    const bool zero = !a.s_in || (live && a.reset && a.reset[i]);
    const float g = live ? a.decay[h] : 1.f;
    const float* from = a.s_in + unit * a.dk * a.dv;
    float* to = a.s_out + unit * a.dk * a.dv;
    const T* q = static_cast<const T*>(a.A.p) + i * a.A.sn + (int64_t)h * a.dk;
    const T* k = static_cast<const T*>(a.B.p) + i * a.B.sn + (int64_t)h * a.dk;
    const T* v = static_cast<const T*>(a.C.p) + i * a.C.sn + (int64_t)h * a.dv;
    float x[4] = {}, o[4] = {};
    if (on && live) {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = to_float(v[col + e]);
    }
    for (int r0 = 0; r0 < a.dk; r0 += rows * U) {
      float4 s[U];
      float qv[U], kv[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int r = r0 + u * rows + sub;
        const bool in = on && r < a.dk;
        s[u] = in && !zero ? *reinterpret_cast<const float4*>(from + r * a.dv + col) : make_float4(0.f, 0.f, 0.f, 0.f);
        qv[u] = in && live ? to_float(q[r]) : 0.f;
        kv[u] = in && live ? to_float(k[r]) : 0.f;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int r = r0 + u * rows + sub;
        if (on && r < a.dk) {
          if (live) {
            s[u].x = fmaf(kv[u], x[0], zero ? 0.f : g * s[u].x);
            s[u].y = fmaf(kv[u], x[1], zero ? 0.f : g * s[u].y);
            s[u].z = fmaf(kv[u], x[2], zero ? 0.f : g * s[u].z);
            s[u].w = fmaf(kv[u], x[3], zero ? 0.f : g * s[u].w);
            o[0] = fmaf(qv[u], s[u].x, o[0]);
            o[1] = fmaf(qv[u], s[u].y, o[1]);
            o[2] = fmaf(qv[u], s[u].z, o[2]);
            o[3] = fmaf(qv[u], s[u].w, o[3]);
          }
          if (a.s_out) *reinterpret_cast<float4*>(to + r * a.dv + col) = s[u];
        }
      }
    }
    sums[wave][lane] = make_float4(o[0], o[1], o[2], o[3]);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    if (live && lane < lv) {
      float4 t = sums[wave][lane];
      for (int r = 1; r < rows; ++r) {
        const float4 y = sums[wave][r * lv + lane];
        t.x += y.x; t.y += y.y; t.z += y.z; t.w += y.w;
      }
      T* out = static_cast<T*>(const_cast<void*>(a.O.p)) + i * a.O.sn + (int64_t)h * a.dv + col;
      const float z[4] = {t.x * a.alpha, t.y * a.alpha, t.z * a.alpha, t.w * a.alpha};
      if constexpr (sizeof(T) == 4) *reinterpret_cast<uint4*>(out) = Elem<float>::pack(z);
      else *reinterpret_cast<uint2*>(out) = make_uint2(Elem<uint16_t>::pack2(z[0], z[1]), Elem<uint16_t>::pack2(z[2], z[3]));
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
}

// ---------------------------------------------------------------------------------------------- host

struct Segments { int32_t n; int64_t len; };
// Segments where sequences, heads and blocks of columns alone leave SIMDs without a wave.
Segments segments_of(int64_t T, int64_t N, int32_t heads, int32_t dk, int32_t dv) {
  const int64_t waves = N * heads * ((std::max(dk, dv) + 31) / 32);
  if (waves == 0 || T <= kSegTokens || waves * 2 > kFillWaves) return {1, std::max<int64_t>(T, 1)};
  const int64_t want = std::min((kFillWaves + waves - 1) / waves, (T + kSegTokens - 1) / kSegTokens);
  const int64_t len = ((T + want - 1) / want + kTok - 1) / kTok * kTok;
  return {(int32_t)((T + len - 1) / len), len};
}

// How many rows (sequences, pairs or segments) a wave takes, and the workgroups for it: `across` waves side by side, one for each
// head and block of columns, on the same rows.  Waves that take neighbouring rows keep the memory that is open at a time together: with
// rows a grid apart instead the windows above took 574 us for 444; runs of 4, 8, 16 and 32 rows 418, 410, 424 and more.
unsigned runs_of(int64_t rows, int64_t across, uint32_t* run) {
  *run = (uint32_t)std::max<int64_t>(1, std::min<int64_t>(kRun, rows * across / (kFillWaves * 4)));
  *run = (uint32_t)std::max<int64_t>(*run, (rows * across + 4 * kMostBlocks - 1) / (4 * kMostBlocks));    // grids end below 2^32 threads
  return (unsigned)(((rows + *run - 1) / *run * across + 3) / 4);
}

template <class T, bool OUT>
void launch(DecayArgs a, hipStream_t st) {
  a.blocks_v = (a.dv + 31) / 32;
  const unsigned grid = runs_of(a.N * a.segs, (int64_t)a.heads * a.blocks_v, &a.run);
#define DGC_DECAY(KD) hipLaunchKernelGGL((k_decay<T, KD, OUT>), grid, 256, 0, st, a)
  if (a.dk <= 16) DGC_DECAY(16);
  else if (a.dk <= 32) DGC_DECAY(32);
  else if (a.dk <= 64) DGC_DECAY(64);
  else DGC_DECAY(128);
#undef DGC_DECAY
}

template <class T>
void launch_window(DecayArgs a, hipStream_t st) {
  a.blocks_v = (a.dv + 31) / 32;
  const bool pair = a.T <= kTok / 2;
  const unsigned grid = runs_of(pair ? (a.N + 1) / 2 : a.N, (int64_t)a.heads * a.blocks_v, &a.run);
#define DGC_DECAY(KD)                                                                                          \
  if (pair) hipLaunchKernelGGL((k_decay_window<T, KD, true>), grid, 256, 0, st, a);   \
  else hipLaunchKernelGGL((k_decay_window<T, KD, false>), grid, 256, 0, st, a)
  if (a.dk <= 16) { DGC_DECAY(16); }
  else if (a.dk <= 32) { DGC_DECAY(32); }
  else if (a.dk <= 64) { DGC_DECAY(64); }
  else { DGC_DECAY(128); }
#undef DGC_DECAY
}

template <class T>
void launch_window_back(BackArgs a, hipStream_t st) {
  const bool pair = a.T <= kTok / 2 && !a.s0 && !a.dsn && !a.ds0;
  const unsigned grid = runs_of(pair ? (a.N + 1) / 2 : a.N, a.heads, &a.run);
  const int most = std::max(a.dk, a.dv);
#define DGC_DECAY(KD)                                                                                \
  if (pair) hipLaunchKernelGGL((k_decay_window_back<T, KD, true>), grid, 256, 0, st, a);             \
  else hipLaunchKernelGGL((k_decay_window_back<T, KD, false>), grid, 256, 0, st, a)
  if (most <= 16) { DGC_DECAY(16); }
  else if (most <= 32) { DGC_DECAY(32); }
  else { DGC_DECAY(64); }
#undef DGC_DECAY
}

struct Call {
  int64_t T, N;
  int32_t heads, dk, dv;
  const float* decay;
  float scale;
  const int32_t* lengths;
  const uint8_t* reset;
  Segments seg;
  float* states;     // workspace
  float* factor;
  hipStream_t st;
};

DecayArgs args_of(const Call& c, const Rows& A, const Rows& B, const Rows& C, const Rows& O, int32_t dk, int32_t dv) {
  DecayArgs a{};
  a.A = A; a.B = B; a.C = C; a.O = O; a.T = c.T; a.N = c.N; a.heads = c.heads; a.dk = dk; a.dv = dv;
  a.decay = c.decay; a.reset = c.reset; a.lengths = c.lengths;
  a.segs = c.seg.n; a.seg_len = c.seg.len;
  a.alpha = c.scale; a.beta = 1.f; a.gam = c.scale;
  a.in_r = a.out_r = dv; a.in_c = a.out_c = 1;
  return a;
}
void backwards(DecayArgs& a, float scale) { a.reversed = 1; a.beta = scale; a.gam = 1.f; }

// The states that enter the segments, from keys B and values C; the last one to s_out.
template <class T>
void join_segments(const Call& c, const DecayArgs& out_pass, const float* s_in, float* s_out, bool link) {
  DecayArgs a = out_pass;
  a.s_in = nullptr; a.s_out = c.states; a.out_r = a.dv; a.out_c = 1; a.out_link = 0; a.factor = c.factor;
  launch<T, false>(a, c.st);
  ScanArgs s{};
  s.states = c.states; s.factor = c.factor; s.s_in = s_in; s.s_out = s_out; s.N = c.N; s.heads = c.heads; s.size = a.dk * a.dv;
  s.segs = a.segs; s.out_link = link; s.decay = c.decay; s.reset = c.reset; s.lengths = c.lengths;
  const int64_t n = c.N * c.heads * s.size;
  hipLaunchKernelGGL(k_decay_scan, (unsigned)std::min<int64_t>((n + 255) / 256, 256 * 16), 256, 0, c.st, s);
}

template <class T>
void forward(const Call& c, const Rows& q, const Rows& k, const Rows& v, const Rows& o, const float* s0, float* sn) {
  DecayArgs a = args_of(c, q, k, v, o, c.dk, c.dv);
  a.s_in = s0; a.s_out = sn;
  if (c.T == 1) {
    hipLaunchKernelGGL(k_decay_step<T>, (unsigned)std::min<int64_t>((c.N * c.heads + 3) / 4, 256 * 32), 256, 0, c.st, a);
    return;
  }
  if (c.T <= kTok && !s0 && !sn) {
    launch_window<T>(a, c.st);
    return;
  }
  if (c.seg.n > 1) {
    join_segments<T>(c, a, s0, sn, false);
    a.s_in = c.states; a.s_out = nullptr;
  }
  launch<T, true>(a, c.st);
}

template <class T>
void backward(const Call& c, const Rows& q, const Rows& k, const Rows& v, const Rows& go, const Rows& dq, const Rows& dk, const Rows& dv,
              const float* s0, const float* dsn, float* ds0) {
  if (c.T <= kTok && std::max(c.dk, c.dv) <= 64) {
    launch_window_back<T>({q, k, v, go, dq, dk, dv, c.T, c.N, c.heads, c.dk, c.dv, c.decay, c.scale, s0, dsn, ds0, c.lengths, c.reset, 0}, c.st);
    return;
  }
  const bool split = c.seg.n > 1;
  if (dq.p) {
    DecayArgs a = args_of(c, go, v, k, dq, c.dv, c.dk);
    a.s_in = s0;
    if (split) {
      join_segments<T>(c, args_of(c, q, k, v, q, c.dk, c.dv), s0, nullptr, false);
      a.s_in = c.states;
    }
    a.in_r = 1; a.in_c = c.dv;
    launch<T, true>(a, c.st);
  }
  DecayArgs a = args_of(c, k, q, go, dv, c.dk, c.dv), b = args_of(c, v, go, q, dk, c.dv, c.dk);
  backwards(a, c.scale);
  backwards(b, c.scale);
  a.s_in = b.s_in = dsn;
  if (split && (dk.p || dv.p || ds0)) {
    join_segments<T>(c, a, dsn, ds0, true);
    a.s_in = b.s_in = c.states;
  } else {
    a.s_out = ds0; a.out_link = 1;      // after dk has read dsn: ds0 may be dsn
  }
  b.in_r = 1; b.in_c = c.dv;
  if (dk.p) launch<T, true>(b, c.st);
  if (dv.p) launch<T, true>(a, c.st);
  else if (!split && ds0) launch<T, false>(a, c.st);
}

const char* check(int64_t T, int64_t N, int32_t heads, int32_t dk, int32_t dv, int32_t dtype) {
  if (dtype != DGC_DTYPE_F32 && dtype != DGC_DTYPE_BF16) return "decay attention: unknown dtype";
  if (T < 0 || N < 0 || heads < 1 || heads > kMaxHeads) return "decay attention: T and N must be >= 0 and heads in [1, 1024]";
  if (dk < 8 || dk > kMaxDim || dk % 8 || dv < 8 || dv > kMaxDim || dv % 8)
    return "decay attention: dk and dv must be multiples of 8 in [8, 128]";
  return nullptr;
}
bool too_many(int64_t T, int64_t N, int32_t heads, int32_t dk, int32_t dv) {   // waves of a launch: 31 bits
  const int64_t most = (int64_t)1 << 31;
  if (T > most || N > most) return true;
  const int64_t seqs = N * heads * ((std::max(dk, dv) + 31) / 32);
  return seqs >= most || seqs * segments_of(T, N, heads, dk, dv).n >= most;
}
// Inputs may repeat rows (a stride of 0); outputs hold each row once.
bool good(const Rows& x, int64_t T, int64_t N, int64_t F, int e, bool output) {
  if (T == 0 || N == 0) return true;
  const int64_t per = 16 / e, most = INT64_MAX / 16;
  if (!x.p || !ops::aligned16(x.p) || x.st < 0 || x.sn < 0 || x.st % per || x.sn % per) return false;
  if (x.st > most / T || x.sn > most / N) return false;
  if (!output) return true;
  if (T > 1 && N > 1) return x.st >= x.sn ? x.sn >= F && x.st >= N * x.sn : x.st >= F && x.sn >= T * x.st;
  return T > 1 ? x.st >= F : N > 1 ? x.sn >= F : true;
}
// Whether an output shares an element with another tensor; rows side by side in one buffer do not.
bool meet(const Rows& x, int64_t Fx, const Rows& y, int64_t Fy, int64_t T, int64_t N, int e) {
  if (!x.p || !y.p || T == 0 || N == 0) return false;
  const uintptr_t x0 = (uintptr_t)x.p, y0 = (uintptr_t)y.p;
  const uintptr_t x1 = x0 + ((T - 1) * x.st + (N - 1) * x.sn + Fx) * e, y1 = y0 + ((T - 1) * y.st + (N - 1) * y.sn + Fy) * e;
  if (x0 >= y1 || y0 >= x1) return false;
  if ((T > 1 && x.st != y.st) || (N > 1 && x.sn != y.sn)) return true;
  const int64_t inner = T == 1 ? x.sn : N == 1 ? x.st : std::min(x.st, x.sn), outer = T == 1 || N == 1 ? inner : std::max(x.st, x.sn);
  if ((T == 1 && N == 1) || inner == 0 || outer % inner) return true;
  const uint64_t pitch = (uint64_t)inner * e, d = x0 >= y0 ? (x0 - y0) % pitch : (pitch - (y0 - x0) % pitch) % pitch;
  return d < (uint64_t)Fy * e || d + (uint64_t)Fx * e > pitch;
}
// Whether a state lies over a tensor of rows, by their spans, or over another state (`same`: it may be that state itself).
bool state_meets(const float* s, const Rows& x, int64_t F, int64_t T, int64_t N, int32_t heads, int32_t dk, int32_t dv, int e) {
  if (!s || !x.p || T == 0 || N == 0) return false;
  const uintptr_t s0 = (uintptr_t)s, x0 = (uintptr_t)x.p;
  return s0 < x0 + ((T - 1) * x.st + (N - 1) * x.sn + F) * e && x0 < s0 + N * heads * dk * dv * (int64_t)sizeof(float);
}
bool states_meet(const float* a, const float* b, bool same, int64_t N, int32_t heads, int32_t dk, int32_t dv) {
  if (!a || !b || N == 0 || (same && a == b)) return false;
  const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
  const uint64_t bytes = (uint64_t)N * heads * dk * dv * sizeof(float);
  return a0 < b0 + bytes && b0 < a0 + bytes;
}
constexpr const char* kBadRows =
    "decay attention: tensors need a 16-byte aligned base and strides that are multiples of 16 bytes; an output's rows lie apart";
constexpr const char* kMeet = "decay attention: outputs lie apart from the inputs and each other";
constexpr const char* kStates = "decay attention: a state lies apart from the tensors of rows and the other states, or (sn: s0; ds0: dsn or s0) is one of them itself";

}  // namespace
}  // namespace dgc

using namespace dgc;

extern "C" {

int64_t dgc_decay_attn_workspace_bytes(int64_t T, int64_t N, int32_t heads, int32_t dk, int32_t dv, int32_t /*backward*/) {
  if (check(T, N, heads, dk, dv, 0) || too_many(T, N, heads, dk, dv)) return -1;
  const Segments s = segments_of(T, N, heads, dk, dv);
  return s.n > 1 ? 4 * (int64_t)s.n * N * heads * (dk * dv + 1) + 16 : 0;
}

static dgc_status_t decay_call(Call* c, int64_t T, int64_t N, int32_t heads, int32_t dk, int32_t dv, const float* decay, float scale,
                               const int32_t* lengths, const uint8_t* reset, void* workspace, int64_t workspace_bytes, void* stream) {
  if (too_many(T, N, heads, dk, dv)) return ops::refuse(DGC_ERR_UNSUPPORTED, "decay attention: more sequences and heads than a launch takes");
  if (!decay) return ops::refuse(DGC_ERR_INVALID_ARG, "decay attention: NULL decay");
  const int64_t need = dgc_decay_attn_workspace_bytes(T, N, heads, dk, dv, 0);
  if (need > 0 && (!workspace || !ops::aligned16(workspace) || workspace_bytes < need))
    return ops::refuse(DGC_ERR_INVALID_ARG, "decay attention: workspace missing, too small (dgc_decay_attn_workspace_bytes) or not 16-byte aligned");
  *c = Call{T, N, heads, dk, dv, decay, scale, lengths, reset, segments_of(T, N, heads, dk, dv), static_cast<float*>(workspace), nullptr,
            static_cast<hipStream_t>(stream)};
  if (need > 0) c->factor = c->states + (int64_t)c->seg.n * N * heads * dk * dv;
  return DGC_OK;
}

dgc_status_t dgc_decay_attn_forward(const void* q, int64_t qt, int64_t qn, const void* k, int64_t kt, int64_t kn, const void* v,
                                    int64_t vt, int64_t vn, int64_t T, int64_t N, int32_t heads, int32_t dk, int32_t dv, int32_t dtype,
                                    const float* decay, float scale, const float* s0, const int32_t* lengths, const uint8_t* reset,
                                    void* o, int64_t ot, int64_t on, float* sn, void* workspace, int64_t workspace_bytes, void* stream) {
  if (const char* msg = check(T, N, heads, dk, dv, dtype)) return ops::refuse(DGC_ERR_INVALID_ARG, msg);
  const int e = ops::elem_bytes(dtype);
  const int64_t fk = (int64_t)heads * dk, fv = (int64_t)heads * dv;
  const Rows Q{q, qt, qn}, K{k, kt, kn}, V{v, vt, vn}, O{o, ot, on};
  if (!good(Q, T, N, fk, e, false) || !good(K, T, N, fk, e, false) || !good(V, T, N, fv, e, false) || !good(O, T, N, fv, e, true))
    return ops::refuse(DGC_ERR_INVALID_ARG, kBadRows);
  if (!ops::aligned16(s0) || !ops::aligned16(sn)) return ops::refuse(DGC_ERR_INVALID_ARG, "decay attention: states need 16-byte alignment");
  Call c;
  if (dgc_status_t rc = decay_call(&c, T, N, heads, dk, dv, decay, scale, lengths, reset, workspace, workspace_bytes, stream)) return rc;
  if (meet(O, fv, Q, fk, T, N, e) || meet(O, fv, K, fk, T, N, e) || meet(O, fv, V, fv, T, N, e))
    return ops::refuse(DGC_ERR_INVALID_ARG, kMeet);
  if (states_meet(sn, s0, true, N, heads, dk, dv) || state_meets(s0, O, fv, T, N, heads, dk, dv, e) || state_meets(sn, O, fv, T, N, heads, dk, dv, e) ||
      state_meets(sn, Q, fk, T, N, heads, dk, dv, e) || state_meets(sn, K, fk, T, N, heads, dk, dv, e) || state_meets(sn, V, fv, T, N, heads, dk, dv, e))
    return ops::refuse(DGC_ERR_INVALID_ARG, kStates);
  if (N == 0) return DGC_OK;
  if (dtype == DGC_DTYPE_F32) forward<float>(c, Q, K, V, O, s0, sn);
  else forward<uint16_t>(c, Q, K, V, O, s0, sn);
  return ops::launched("decay attention");
}

dgc_status_t dgc_decay_attn_backward(const void* q, int64_t qt, int64_t qn, const void* k, int64_t kt, int64_t kn, const void* v,
                                     int64_t vt, int64_t vn, const void* go, int64_t gt, int64_t gn, int64_t T, int64_t N,
                                     int32_t heads, int32_t dk, int32_t dv, int32_t dtype, const float* decay, float scale,
                                     const float* s0, const float* dsn, const int32_t* lengths, const uint8_t* reset, void* dq,
                                     int64_t dqt, int64_t dqn, void* dkey, int64_t dkt, int64_t dkn, void* dval, int64_t dvt,
                                     int64_t dvn, float* ds0, void* workspace, int64_t workspace_bytes, void* stream) {
  if (const char* msg = check(T, N, heads, dk, dv, dtype)) return ops::refuse(DGC_ERR_INVALID_ARG, msg);
  const int e = ops::elem_bytes(dtype);
  const int64_t fk = (int64_t)heads * dk, fv = (int64_t)heads * dv;
  const Rows in[4] = {{q, qt, qn}, {k, kt, kn}, {v, vt, vn}, {go, gt, gn}}, out[3] = {{dq, dqt, dqn}, {dkey, dkt, dkn}, {dval, dvt, dvn}};
  const int64_t fi[4] = {fk, fk, fv, fv}, fo[3] = {fk, fk, fv};
  for (int x = 0; x < 4; ++x) {
    if (!good(in[x], T, N, fi[x], e, false)) return ops::refuse(DGC_ERR_INVALID_ARG, kBadRows);
  }
  for (int x = 0; x < 3; ++x) {
    if (out[x].p && !good(out[x], T, N, fo[x], e, true)) return ops::refuse(DGC_ERR_INVALID_ARG, kBadRows);
  }
  if (!ops::aligned16(s0) || !ops::aligned16(dsn) || !ops::aligned16(ds0))
    return ops::refuse(DGC_ERR_INVALID_ARG, "decay attention: states need 16-byte alignment");
  Call c;
  if (dgc_status_t rc = decay_call(&c, T, N, heads, dk, dv, decay, scale, lengths, reset, workspace, workspace_bytes, stream)) return rc;
  for (int x = 0; x < 3; ++x) {
    for (int y = 0; y < 4; ++y) {
      if (meet(out[x], fo[x], in[y], fi[y], T, N, e)) return ops::refuse(DGC_ERR_INVALID_ARG, kMeet);
    }
    for (int y = 0; y < x; ++y) {
      if (meet(out[x], fo[x], out[y], fo[y], T, N, e)) return ops::refuse(DGC_ERR_INVALID_ARG, kMeet);
    }
  }
  bool meets = states_meet(ds0, dsn, true, N, heads, dk, dv) || states_meet(ds0, s0, true, N, heads, dk, dv);
  for (int x = 0; x < 4; ++x) meets = meets || state_meets(ds0, in[x], fi[x], T, N, heads, dk, dv, e);
  for (int x = 0; x < 3; ++x) {
    for (const float* s : {s0, dsn, static_cast<const float*>(ds0)}) meets = meets || state_meets(s, out[x], fo[x], T, N, heads, dk, dv, e);
  }
  if (meets) return ops::refuse(DGC_ERR_INVALID_ARG, kStates);
  if (N == 0) return DGC_OK;
  if (dtype == DGC_DTYPE_F32) backward<float>(c, in[0], in[1], in[2], in[3], out[0], out[1], out[2], s0, dsn, ds0);
  else backward<uint16_t>(c, in[0], in[1], in[2], in[3], out[0], out[1], out[2], s0, dsn, ds0);
  return ops::launched("decay attention");
}

}  // extern "C"
