// Device helpers of the softmax attention kernels: matrix tiles of three kinds, one interface; and the host's rules, which kernel and how many parts.
//
// A product c += x y on the matrix unit takes x as rows (a lane holds KE consecutive contraction indices of its row) and
// y as columns, and leaves c with a column a lane and NR rows in its registers.  All kernels here are built on one fact: what a
// product left, c's rows in a lane's registers, is just what the next product wants of its right operand when those rows are summed
// over, so scores become probabilities and meet the values without leaving their lane.  The left operand of that next product then
// comes across its rows: out of LDS, by the transposing read for bf16 and element by element for fp32.
//   Wide  bf16, 32 x 32 results (v_mfma_f32_32x32x16_bf16)
//   Small bf16, 16 x 16 results (v_mfma_f32_16x16x16_bf16): short windows, where 32 x 32 would be half empty
//   Full  fp32, 16 x 16 results (four v_mfma_f32_16x16x4_f32 a step): products as exact as fp32 arithmetic
#pragma once

#include "dgc_ops.h"

namespace dgc {
namespace attn {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t wordx4 __attribute__((ext_vector_type(4)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) shortx4* lds_shortx4;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMaxHeads = 1024, kMaxDim = 128, kMaxReach = 1024, kMaxBuckets = 256, kMaxSplits = 1024;

struct Rows {          // row (t, i) at p + t st + i sn, in elements
  const void* p;
  int64_t st, sn;
};

// What the calls have in common; a pointer that is not wanted is nullptr.
struct Args {
  Rows q, k, v, o, go, dq, dk, dv;
  int64_t N;
  int32_t Tq, Tk, heads, group, d;     // group: heads that share a key head
  int32_t causal, buckets, reach;
  float scale;
  const int32_t *first, *lengths;
  const uint8_t *keep, *map;
  const float* bias;
  float* lse;          // [N][heads][Tq]
  float* delta;        // the same
  int32_t* odd;        // whether a workgroup's work is to be done again by the kernel that keeps what is not finite apart
  float* part;         // partial sums of the bias' gradient: [heads][slots][kind of table]
  int32_t slots;       // workgroups (windows: waves) of a head
  int32_t splits;      // few queries: parts of the keys
  int32_t head_parts, row_parts;       // parts of the heads and queries that a key's gradients are summed over
  float* joint;        // few queries: the parts' outputs, not divided, and statistics; keys: the parts' gradients
};

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }   // v_exp_f32: 1 ulp, 0 for -inf
// Biases and statistics of the type's lowest value or near it: scores have no bits left beside them, and are to lose them everywhere.  The same of large
// scores: (s - off) log2e by one multiply-add is off by 2^-22 of off, here 0.25, and by more than fp32 has exponents from 10^9 on.
__device__ __forceinline__ bool far_off(float off) { return fabsf(off) > 1048576.f; }
// e^(x - off); off is a maximum, -inf if there is nothing.
__device__ __forceinline__ float weight_of(float x, float off) { return exp2_((x - (off == -__builtin_inff() ? 0.f : off)) * kLog2e); }
__device__ __forceinline__ float log_sum(float top, float sum) { return sum == 0.f ? -__builtin_inff() : fmaf(__builtin_amdgcn_logf(sum), kLn2, top); }      // the sum has a term of 1: its logarithm is off by 2^-23
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const bf16x2 v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ bool odd_bf16(uint32_t w) {   // one of two bf16 numbers is an infinity or NaN
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}
__device__ __forceinline__ bool odd_f32(uint32_t w) { return (w & 0x7f800000u) == 0x7f800000u; }

__device__ __forceinline__ uint4 kept(uint4 w, bool ok) { return make_uint4(ok ? w.x : 0u, ok ? w.y : 0u, ok ? w.z : 0u, ok ? w.w : 0u); }

struct Wide {
  typedef uint16_t E;
  typedef uint4 Frag;
  typedef floatx16 Acc;
  static constexpr int M = 32, NR = 16, KE = 8, KSM = 2, SUBS = 2;
  static constexpr bool kExact = false;
  static __device__ __forceinline__ int col(int lane) { return lane & 31; }
  static __device__ __forceinline__ int sub(int lane) { return lane >> 5; }
  static constexpr __device__ __forceinline__ int row(int r) { return 8 * (r >> 2) + (r & 3); }      // of lane 0; 4 sub more of another
  // The row that element e of a fragment packed from rows, step s, stands for.
  static __device__ __forceinline__ int index(int s, int e, int lane) { return 16 * s + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3); }
  static __device__ __forceinline__ Acc mma(Frag a, Frag b, Acc c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ Frag zero() { return make_uint4(0, 0, 0, 0); }
  static __device__ __forceinline__ Frag rows(const E* p, int pitch, int s, int lane) {     // p: row 0 of the tile
    return *reinterpret_cast<const uint4*>(p + (lane & 31) * pitch + 16 * s + 8 * (lane >> 5));
  }
  static __device__ __forceinline__ Frag across(const E* p, int pitch, int s, int dt, int lane) {
    const E* at = p + (16 * s + 4 * (lane >> 5) + ((lane & 15) >> 2)) * pitch + 32 * dt + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    const shortx4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4)at);
    const shortx4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4)(at + 8 * pitch));
    const uint2 x = __builtin_bit_cast(uint2, a), y = __builtin_bit_cast(uint2, b);
    return make_uint4(x.x, x.y, y.x, y.y);
  }
  static __device__ __forceinline__ Frag pack(const Acc& c, int s) {
    return make_uint4(pack2(c[8 * s], c[8 * s + 1]), pack2(c[8 * s + 2], c[8 * s + 3]), pack2(c[8 * s + 4], c[8 * s + 5]), pack2(c[8 * s + 6], c[8 * s + 7]));
  }
  static __device__ __forceinline__ Frag upto(Frag f, int s, int lane, int lo, int hi) {   // rows outside [lo, hi] zero
    uint32_t w[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int i = index(s, e, lane);
      if (i < lo || i > hi) w[e / 2] &= e & 1 ? 0xffffu : 0xffff0000u;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ bool odd(uint4 w) { return odd_bf16(w.x) || odd_bf16(w.y) || odd_bf16(w.z) || odd_bf16(w.w); }
};

struct Small {
  typedef uint16_t E;
  typedef uint2 Frag;
  typedef floatx4 Acc;
  static constexpr int M = 16, NR = 4, KE = 4, KSM = 1, SUBS = 4;
  static constexpr bool kExact = false;
  static __device__ __forceinline__ int col(int lane) { return lane & 15; }
  static __device__ __forceinline__ int sub(int lane) { return lane >> 4; }
  static constexpr __device__ __forceinline__ int row(int r) { return r; }
  static __device__ __forceinline__ int index(int s, int e, int lane) { return 16 * s + 4 * (lane >> 4) + e; }
  static __device__ __forceinline__ Acc mma(Frag a, Frag b, Acc c) {
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(shortx4, a), __builtin_bit_cast(shortx4, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ Frag zero() { return make_uint2(0, 0); }
  static __device__ __forceinline__ Frag load(const E* p) { return *reinterpret_cast<const uint2*>(p); }
  static __device__ __forceinline__ void store(E* p, Frag f) { *reinterpret_cast<uint2*>(p) = f; }
  static __device__ __forceinline__ Frag rows(const E* p, int pitch, int s, int lane) { return load(p + (lane & 15) * pitch + 16 * s + 4 * (lane >> 4)); }
  static __device__ __forceinline__ Frag across(const E* p, int pitch, int s, int dt, int lane) {
    const E* at = p + (16 * s + 4 * (lane >> 4) + ((lane & 15) >> 2)) * pitch + 16 * dt + 4 * (lane & 3);
    const shortx4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4)at);
    return __builtin_bit_cast(uint2, a);
  }
  static __device__ __forceinline__ Frag pack(const Acc& c, int) { return make_uint2(pack2(c[0], c[1]), pack2(c[2], c[3])); }
  static __device__ __forceinline__ Frag upto(Frag f, int s, int lane, int lo, int hi) {
    uint32_t w[2] = {f.x, f.y};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = index(s, e, lane);
      if (i < lo || i > hi) w[e / 2] &= e & 1 ? 0xffffu : 0xffff0000u;
    }
    return make_uint2(w[0], w[1]);
  }
  static __device__ __forceinline__ bool odd(uint2 w) { return odd_bf16(w.x) || odd_bf16(w.y); }
  static __device__ __forceinline__ float dot(Frag a, Frag b) {
    float s = 0.f;
    const uint32_t x[2] = {a.x, a.y}, y[2] = {b.x, b.y};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      s = fmaf(__uint_as_float(x[i] << 16), __uint_as_float(y[i] << 16), s);
      s = fmaf(__uint_as_float(x[i] & 0xffff0000u), __uint_as_float(y[i] & 0xffff0000u), s);
    }
    return s;
  }
};

struct Full {
  typedef float E;
  typedef uint4 Frag;
  typedef floatx4 Acc;
  static constexpr int M = 16, NR = 4, KE = 4, KSM = 1, SUBS = 4;
  static constexpr bool kExact = true;        // the difference of exponents is taken before it is multiplied
  static __device__ __forceinline__ int col(int lane) { return lane & 15; }
  static __device__ __forceinline__ int sub(int lane) { return lane >> 4; }
  static constexpr __device__ __forceinline__ int row(int r) { return r; }
  static __device__ __forceinline__ int index(int s, int e, int lane) { return 16 * s + 4 * (lane >> 4) + e; }
  static __device__ __forceinline__ Acc mma(Frag a, Frag b, Acc c) {
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
  }
  static __device__ __forceinline__ Frag zero() { return make_uint4(0, 0, 0, 0); }
  static __device__ __forceinline__ Frag load(const E* p) { return *reinterpret_cast<const uint4*>(p); }
  static __device__ __forceinline__ void store(E* p, Frag f) { *reinterpret_cast<uint4*>(p) = f; }
  static __device__ __forceinline__ Frag rows(const E* p, int pitch, int s, int lane) { return load(p + (lane & 15) * pitch + 16 * s + 4 * (lane >> 4)); }
  static __device__ __forceinline__ Frag across(const E* p, int pitch, int s, int dt, int lane) {
    const uint32_t* at = reinterpret_cast<const uint32_t*>(p) + (16 * s + 4 * (lane >> 4)) * pitch + 16 * dt + (lane & 15);
    return make_uint4(at[0], at[pitch], at[2 * pitch], at[3 * pitch]);
  }
  static __device__ __forceinline__ Frag pack(const Acc& c, int) {
    return make_uint4(__float_as_uint(c[0]), __float_as_uint(c[1]), __float_as_uint(c[2]), __float_as_uint(c[3]));
  }
  static __device__ __forceinline__ Frag upto(Frag f, int s, int lane, int lo, int hi) {
    uint32_t w[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int i = index(s, e, lane);
      if (i < lo || i > hi) w[e] = 0;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static __device__ __forceinline__ bool odd(uint4 w) { return odd_f32(w.x) || odd_f32(w.y) || odd_f32(w.z) || odd_f32(w.w); }
  static __device__ __forceinline__ float dot(Frag a, Frag b) {
    float s = __uint_as_float(a.x) * __uint_as_float(b.x);
    s = fmaf(__uint_as_float(a.y), __uint_as_float(b.y), s);
    s = fmaf(__uint_as_float(a.z), __uint_as_float(b.z), s);
    return fmaf(__uint_as_float(a.w), __uint_as_float(b.w), s);
  }
};

// What all lanes of a wave agree on, as the compiler cannot know.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Sums and maxima over the lanes that hold rows of one column.
template <int SUBS>
__device__ __forceinline__ float column_max(float x) {
  if constexpr (SUBS == 4) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  }
  const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
template <int SUBS>
__device__ __forceinline__ float column_sum(float x) {
  if constexpr (SUBS == 4) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  }
  const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}
// What one lane of a wave writes to LDS and another reads: the unit works in order, the compiler is told to.
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ float wave_sum(float x) {     // in one order
  for (int m = 1; m < 64; m *= 2) x += __shfl_xor(x, m);
  return x;
}

// Sequence n: its tokens, the position of its first query, and the queries [lo, hi) that are among its tokens.
struct Seq {
  int64_t at;
  int len, lo, hi;
  __device__ __forceinline__ Seq(const Args& a, int64_t n) {
    at = a.first ? (int64_t)a.first[n] : (int64_t)(a.Tk - a.Tq);
    len = a.lengths ? min(max(a.lengths[n], 0), a.Tk) : a.Tk;
    lo = (int)min(max(-at, (int64_t)0), (int64_t)a.Tq);
    hi = (int)min(max((int64_t)len - at, (int64_t)0), (int64_t)a.Tq);
  }
};

// The bias of head h at a distance (query's position minus key's).
__device__ __forceinline__ float bias_at(const Args& a, int h, int64_t away) {
  const int c = (int)min(max(away, -(int64_t)a.reach), (int64_t)a.reach) + a.reach;
  return a.bias[(int64_t)h * a.buckets + min((int)a.map[c], a.buckets - 1)];
}

// What a product left as the right operand of the next, which sums over its rows.
template <class Tl>
struct Packed {
  typename Tl::Frag f[Tl::KSM];
  __device__ __forceinline__ explicit Packed(const typename Tl::Acc& c) {
#pragma unroll
    for (int s = 0; s < Tl::KSM; ++s) f[s] = Tl::pack(c, s);
  }
  __device__ __forceinline__ explicit Packed(typename Tl::Frag x) { f[0] = x; }
};

// acc += left^T right for M rows of left, which lie in LDS.
template <class Tl, int DT>
__device__ __forceinline__ void gather(typename Tl::Acc (&acc)[DT], const typename Tl::E* left, int pitch, const Packed<Tl>& right, int lane) {
#pragma unroll
  for (int s = 0; s < Tl::KSM; ++s) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) acc[dt] = Tl::mma(Tl::across(left, pitch, s, dt, lane), right.f[s], acc[dt]);
  }
}
// The same where a zero of `right` may meet something in left that is not finite: column c takes only the rows [lo(c), hi(c)] that it sees, one
// column after the other.
template <class Tl, int DT, class Lo, class Hi>
__device__ __forceinline__ void gather_seen(typename Tl::Acc (&acc)[DT], const typename Tl::E* left, int pitch, const Packed<Tl>& right, int lane, Lo lo, Hi hi) {
  asm volatile("" : "+v"(lane));      // this is rare: nothing of it is to be held in registers meanwhile
#pragma unroll
  for (int s = 0; s < Tl::KSM; ++s) {
    for (int c = 0; c < Tl::M; ++c) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        typename Tl::Acc t = (typename Tl::Acc)(0.f);
        t = Tl::mma(Tl::upto(Tl::across(left, pitch, s, dt, lane), s, lane, lo(c), hi(c)), right.f[s], t);
#pragma unroll
        for (int r = 0; r < Tl::NR; ++r) acc[dt][r] = Tl::col(lane) == c ? acc[dt][r] + t[r] : acc[dt][r];
      }
    }
  }
}

// A lane's column of an [d x M] result, four consecutive elements at a time, times `by`, into a row of a tensor.
template <class Tl, int DT>
__device__ __forceinline__ void store_column(typename Tl::E* row, const typename Tl::Acc (&acc)[DT], float by, int d, int lane) {
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
    for (int r = 0; r < Tl::NR; r += 4) {
      const int c = dt * Tl::M + Tl::row(r) + 4 * Tl::sub(lane);
      if (c >= d) continue;
      const float x[4] = {acc[dt][r] * by, acc[dt][r + 1] * by, acc[dt][r + 2] * by, acc[dt][r + 3] * by};
      if constexpr (sizeof(typename Tl::E) == 2) *reinterpret_cast<uint2*>(row + c) = make_uint2(pack2(x[0], x[1]), pack2(x[2], x[3]));
      else *reinterpret_cast<float4*>(row + c) = make_float4(x[0], x[1], x[2], x[3]);
    }
  }
}

// The same in fp32, into a row of its own.
template <class Tl, int DT>
__device__ __forceinline__ void store_sums(float* row, const typename Tl::Acc (&acc)[DT], float by, int d, int lane) {
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
    for (int r = 0; r < Tl::NR; r += 4) {
      const int c = dt * Tl::M + Tl::row(r) + 4 * Tl::sub(lane);
      if (c < d) *reinterpret_cast<float4*>(row + c) = make_float4(acc[dt][r] * by, acc[dt][r + 1] * by, acc[dt][r + 2] * by, acc[dt][r + 3] * by);
    }
  }
}

// A tile of rows on its way from memory to LDS by a workgroup of 256: 16 bytes a thread and step; rows that are not `in` are zero.
template <class E, int ROWS, int KS>
struct Stage {
  static constexpr int PER = 16 / sizeof(E), CPR = KS * 16 / PER, N = (ROWS * CPR + 255) / 256;
  uint4 w[N];
  uint32_t off[N];      // bytes from the tile's first row
  bool near, has[N];    // the tile spans less than 2^31 bytes; this chunk is one of the rows'
  static __device__ __forceinline__ int row(int i) { return (int)(threadIdx.x + 256 * i) / CPR; }
  __device__ __forceinline__ void init(int64_t st, int d) {
    near = st < (int64_t)(((uint64_t)1 << 31) / (ROWS * sizeof(E)));
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int x = (int)((threadIdx.x + 256 * i) % CPR) * PER;
      off[i] = (uint32_t)((row(i) * (uint64_t)st + x) * sizeof(E));
      has[i] = (ROWS * CPR % 256 == 0 || row(i) < ROWS) && x < d;
      w[i] = make_uint4(0, 0, 0, 0);
    }
  }
  // A whole tile from its first row on: an address that the workgroup has in common, and a thread's own 32 bits.
  __device__ __forceinline__ void fetch_all(const E* tile) {
    if constexpr (256 % CPR == 0 && ROWS * CPR % 256 == 0) {      // a thread's chunks have their columns in common
      if (has[0]) {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(tile) + off[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (has[i]) w[i] = *reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(tile) + off[i]);
      }
    }
  }
  template <class In>
  __device__ __forceinline__ void fetch(const E* base, int64_t st, int row0, In in) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int x = (int)((threadIdx.x + 256 * i) % CPR) * PER;
      w[i] = has[i] && in(row0 + row(i)) ? *reinterpret_cast<const uint4*>(base + (int64_t)(row0 + row(i)) * st + x) : make_uint4(0, 0, 0, 0);
    }
  }
  __device__ __forceinline__ void put(E* lds, int pitch) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int x = (int)((threadIdx.x + 256 * i) % CPR) * PER;
      if (ROWS * CPR % 256 == 0 || row(i) < ROWS) *reinterpret_cast<uint4*>(lds + row(i) * pitch + x) = w[i];
    }
  }
  template <class Tl>
  __device__ __forceinline__ bool odd() const {
    bool f = false;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if constexpr (sizeof(E) == 2) f = f || odd_bf16(w[i].x) || odd_bf16(w[i].y) || odd_bf16(w[i].z) || odd_bf16(w[i].w);
      else f = f || odd_f32(w[i].x) || odd_f32(w[i].y) || odd_f32(w[i].z) || odd_f32(w[i].w);
    }
    return f;
  }
};

// The bias by distance in LDS, past its reach by as much as a tile that is not far off as a whole can be, so that the tiles' places need no limits.
constexpr int kPast = 96;
struct BiasTable {
  int from, size;
  __device__ __forceinline__ explicit BiasTable(const Args& a) : from((a.causal ? 0 : -a.reach) - kPast), size(a.reach + kPast + 1 - from) {}
  // By distance, or (turned) from the farthest to the nearest: a lane's entries then ascend with its keys.
  __device__ __forceinline__ void fill(const Args& a, float* table, int h, bool turned) const {
    for (int x = threadIdx.x; x < size; x += 256) table[turned ? size - 1 - x : x] = bias_at(a, h, from + x);
  }
};

template <class Tl, int KS>
struct Geometry {
  static constexpr int DT = (KS * 16 + Tl::M - 1) / Tl::M;                    // row tiles of a head
  static constexpr int P = DT * Tl::M + 16 / (int)sizeof(typename Tl::E);     // pitch of rows in LDS: 16 bytes more, so that rows begin in other banks
  static constexpr int NT = Tl::M == 32 && KS >= 8 ? 1 : 2;                   // tiles of M rows on their way at a time, as registers allow
};

// Host side.  The form of a forward pass goes by its lengths alone.
enum Form { kWindow, kFew, kLong };
inline Form form_of(int64_t Tq, int64_t Tk) { return Tk <= 64 ? kWindow : Tq <= 16 ? kFew : kLong; }
// Backward: windows of up to 32 keys whose queries stand at one position, up to 64 wide, with up to four heads to a key head, have a kernel of
// their own.
inline bool takes_window_back(int64_t Tk, int32_t d, int32_t group, bool first) { return Tk <= 32 && d <= 64 && group <= 4 && !first; }
// Entries of a workgroup's table of the bias' gradient by distance, and the distance of the first: beyond `reach` by a tile, so that a tile
// that is not far off as a whole needs no limit.
constexpr int kTile = 64;
inline __host__ __device__ int table_from(int32_t reach, int32_t causal) { return causal ? 0 : -(reach + 2 * kTile); }
inline __host__ __device__ int table_size(int32_t reach, int32_t causal) { return reach + 2 * kTile - table_from(reach, causal); }
// Workgroups of k_attn_dq that the card holds at a time: two a CU as bf16 tiles and wide heads need registers, three or four in fp32 (1000 x 200 tokens, 4 heads of
// 32: 802 us with 1024, 863 with 768, 984 with 512, 845 with 4096; 16 x 1001, 8 of 64: 1107 us with 768, 1154 with 1024, 1169 with 512).
inline int at_once(bool f32, int32_t d) { return !f32 || d > 64 ? 512 : d > 32 ? 768 : 1024; }
// Workgroups (windows: waves) that share a head's queries where the bias' gradient is wanted: as many as the card holds at a time, each of them leaves a table.
inline int back_slots(bool window, int64_t N, int64_t heads, int64_t kvs, int64_t blocks, int at_once) {
  const int64_t most = window ? (256 * 16 + kvs - 1) / kvs : (at_once + heads - 1) / heads, all = window ? N : N * blocks;
  return (int)(all < most ? all : most);
}
// Where keys have too few workgroups to fill the card, their gradients are summed in parts: of the heads that share them first, then of the queries,
// 256 at least.
struct Parts {
  int32_t heads, rows;
};
inline Parts key_parts(int64_t Tq, int64_t Tk, int64_t N, int64_t heads, int64_t kvs, bool f32) {
  const int64_t all = N * kvs * ((Tk + (f32 ? 63 : 127)) / (f32 ? 64 : 128)), group = heads / kvs;
  int64_t want = all ? (1024 + all - 1) / all : 1;
  if (all >= 512) want = 1;
  Parts p{1, 1};
  for (int64_t g = 2; g <= group && g <= 2 * want; ++g) {
    if (group % g == 0) p.heads = (int32_t)g;
  }
  want = (want + p.heads - 1) / p.heads;
  if (all >= 512) p.heads = 1;
  p.rows = (int32_t)(want < Tq / 256 ? want : Tq / 256);
  if (p.rows < 1) p.rows = 1;
  return p;
}
inline unsigned bias_bytes(const Args& a) { return a.bias ? 4 * (unsigned)((a.causal ? a.reach : 2 * a.reach) + 2 * kPast + 1) : 0; }
// Windows backward: whole rows of `together` neighbouring heads of `seqs` sequences a workgroup, four sequences and heads or eight at a time; `slots`
// workgroups a group of heads, each of which leaves `tables` tables of the bias' gradient a head.
struct WindowPlan {
  int32_t together, seqs, groups, slots, tables;
};
inline WindowPlan plan_windows(int64_t N, int64_t heads, int64_t d, int e) {
  WindowPlan p{1, 1, 1, 1, 1};
  while (p.together < 8 && 2 * p.together <= heads && 2 * p.together * d * e <= 256) p.together *= 2;
  p.seqs = p.together < 4 ? 4 / p.together : 1;
  p.groups = (int32_t)((heads + p.together - 1) / p.together);
  p.tables = p.together < 4 ? 4 / p.together : 1;
  const int64_t blocks = (N + p.seqs - 1) / p.seqs, most = (1024 + p.groups - 1) / p.groups;
  p.slots = (int32_t)(blocks < most ? blocks : most);
  return p;
}
void attn_forward_f32(const Args& a, hipStream_t st);
void attn_forward_bf16(const Args& a, hipStream_t st);
void attn_backward_f32(const Args& a, float* dbias, hipStream_t st);
void attn_backward_bf16(const Args& a, float* dbias, hipStream_t st);

}  // namespace attn
}  // namespace dgc
