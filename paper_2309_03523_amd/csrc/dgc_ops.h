// Shared by the kernels that work on plain row-major tensors (norm, linear, decaying attention): 16-byte
// vectors of either element type, and the host checks of pitches, alignment and overlap.
#pragma once

#include "dgc_internal.h"

namespace dgc {
namespace ops {

// Element types: float, or bfloat16 carried as uint16_t (its bits are the top half of a float's).
template <class T> struct Elem;
template <> struct Elem<float> {
  static constexpr int kPer = 4;   // elements of a 16-byte vector
  static __device__ __forceinline__ void unpack(uint4 u, float* x) {
    x[0] = __uint_as_float(u.x); x[1] = __uint_as_float(u.y); x[2] = __uint_as_float(u.z); x[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 pack(const float* x) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
  static __device__ __forceinline__ float one(float x) { return x; }
};
template <> struct Elem<uint16_t> {
  static constexpr int kPer = 8;
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  static __device__ __forceinline__ uint32_t pack2(float a, float b) {   // to the nearest, ties to even
    const bf16x2 v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
  }
  static __device__ __forceinline__ void unpack(uint4 u, float* x) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float* x) {
    return make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
  }
  static __device__ __forceinline__ uint16_t one(float x) { return __builtin_bit_cast(uint16_t, (__bf16)x); }
};

// The vector that starts at column `col` (a multiple of kPer) of a row: zeros in the columns from F on.  A vector with
// a column below F is read whole: pitches are multiples of 16 bytes, so it lies within the row's pitch.
template <class T>
__device__ __forceinline__ void load_vec(const T* row, int col, int F, float* x) {
  constexpr int VN = Elem<T>::kPer;
  if (col < F) {
    Elem<T>::unpack(*reinterpret_cast<const uint4*>(row + col), x);
    if (col + VN > F) {
#pragma unroll
      for (int i = 0; i < VN; ++i) x[i] = col + i < F ? x[i] : 0.f;
    }
  } else {
#pragma unroll
    for (int i = 0; i < VN; ++i) x[i] = 0.f;
  }
}
template <class T>
__device__ __forceinline__ void store_vec(T* row, int col, int F, const float* x) {   // columns from F on stay as they are
  constexpr int VN = Elem<T>::kPer;
  if (col + VN <= F) {
    *reinterpret_cast<uint4*>(row + col) = Elem<T>::pack(x);
  } else {
#pragma unroll
    for (int i = 0; i < VN; ++i) {
      if (col + i < F) row[col + i] = Elem<T>::one(x[i]);
    }
  }
}

// ---- host
inline int elem_bytes(int32_t dtype) { return dtype == DGC_DTYPE_F32 ? 4 : 2; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
inline dgc_status_t refuse(dgc_status_t code, const char* msg) {
  try { set_thread_error(msg); } catch (...) {}   // no exception leaves a C entry
  return code;
}
inline dgc_status_t launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e == hipSuccess) return DGC_OK;
  try { set_thread_error(std::string(what) + ": " + hipGetErrorString(e)); } catch (...) {}
  return DGC_ERR_DEVICE;
}
// A row-major tensor of R rows of F elements: pitch and alignment as the header's conventions say.
inline bool good_rows(const void* p, int64_t R, int64_t F, int64_t ld, int esz) {
  return R == 0 || (p && aligned16(p) && ld >= F && ld % (16 / esz) == 0 && ld <= INT64_MAX / 8 / (R > 0 ? R : 1));
}
// Whether two such tensors share an element.  Of tensors of one pitch, columns that lie side by side do not.
inline bool share(const void* a, int64_t lda, int ea, int64_t Fa, const void* b, int64_t ldb, int eb, int64_t Fb, int64_t R) {
  if (!a || !b || R == 0) return false;
  const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
  const uint64_t pa = (uint64_t)lda * ea, pb = (uint64_t)ldb * eb;
  const uint64_t wa = (uint64_t)Fa * ea, wb = (uint64_t)Fb * eb;
  if (a0 >= b0 + (R - 1) * pb + wb || b0 >= a0 + (R - 1) * pa + wa) return false;
  if (pa != pb) return true;
  const uint64_t d = a0 >= b0 ? (a0 - b0) % pa : (pa - (b0 - a0) % pa) % pa;   // where a row of a starts in one of b
  return d < wb || d + wa > pa;
}
// The same for tensors of different numbers of rows, by their spans alone.
inline bool span_shared(const void* a, int64_t lda, int ea, int64_t Fa, int64_t Ra, const void* b, int64_t ldb, int eb, int64_t Fb, int64_t Rb) {
  if (!a || !b || Ra == 0 || Rb == 0) return false;
  const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
  return a0 < b0 + ((Rb - 1) * ldb + Fb) * eb && b0 < a0 + ((Ra - 1) * lda + Fa) * ea;
}
inline bool same_place(const void* a, int64_t lda, const void* b, int64_t ldb) { return a == b && lda == ldb; }

}  // namespace ops
}  // namespace dgc
