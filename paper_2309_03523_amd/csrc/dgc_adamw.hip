// One AdamW step over many tensors in one launch.  For every parameter, with t the number of the step:
//
//   m <- b1 m + (1 - b1) g,  v <- b2 v + (1 - b2) g^2,  p <- p - lr (m c1 / (sqrt(v) c2 + eps) + decay p),   c1 = 1 / (1 - b1^t),  c2 = (1 - b2^t)^-1/2
//
// What bounds it: memory, 28 bytes a parameter in fp32, 16.06 with bf16 parameters and gradients, fp32 masters and 8-bit states.  A wave
// takes 256 parameters at a time, four neighbours a lane, and a workgroup 4 such blocks a wave, all loads before the first use: 53 million
// parameters in fp32 in 292 us, 5.1 TB/s; 99 million in the other form in 328 to 338 us, 4.8 TB/s (a card's first 40 passes take 340 to 440); the 12 tensors of a small block in 5 us, a call.
//
// States in 8 bits: m, and r = sqrt(v), as e4m3 numbers times a power of two for each 256 of them: the least with which the largest is at most
// 448, e4m3's largest.  A power of two makes that division exact.  The root and not v is held: it spans half the exponents, and one below the least e4m3
// number is raised to it, so no step divides by a root that was lost.  A number is off by at most 2^-4 of itself, or 2^-10 of the scale, a root that is
// raised by up to 2^-9 of the scale; that is
// what 8 bits hold, and the step itself is taken with the states before they are rounded.
// All arithmetic is fp32, one operation after the other without fusing, so a state's code is a function of its inputs
// that can be computed anywhere.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <utility>
#include <vector>

#include "dgc_ops.h"

struct dgc_adamw {
  int bits = 32, device = 0;
  int32_t tensors = 0;
  int64_t chunks = 0;
  void* memory = nullptr;      // one allocation: the tensors, the chunks, the factors of a step
};

namespace dgc {
namespace {

constexpr int kBlock = 256, kBlocks = 16, kChunk = kBlock * kBlocks;     // parameters of a wave's step, and of a workgroup

struct Tensor {
  void* p;
  const void* g;
  float* master;
  void *m, *v;
  float *m_scale, *v_scale;
  int64_t ldp, ldg, ldmaster, total;     // total: rows times the states' pitch
  int32_t F, pitch, bf16;
  float decay;
  int32_t flat;                          // every row at the states' pitch, without columns behind F
};
struct Chunk {
  int32_t tensor;
  uint32_t index;       // of kChunk elements
};
struct Factors {
  float lr, c1, c2;
};
struct StepArgs {
  const Tensor* tensors;
  const Chunk* chunks;
  const Factors* device;      // or nullptr: these
  Factors host;
  float b1, a1, b2, a2, eps;
};

template <int CTRL>
__device__ __forceinline__ float lane_max(float x) {
  return fmaxf(x, __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), CTRL, 0xf, 0xf, true)));
}
__device__ __forceinline__ float wave_max(float x) {      // of numbers >= 0
  x = lane_max<0xB1>(x);       // quad_perm 1 0 3 2
  x = lane_max<0x4E>(x);       // quad_perm 2 3 0 1
  x = lane_max<0x141>(x);      // row_half_mirror
  x = lane_max<0x140>(x);      // row_mirror
  auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

// Four numbers of a row from column c on; those from F on are zero.
__device__ __forceinline__ void load4(const float* row, int c, int F, float (&x)[4]) {
  if (c + 4 <= F) {
    const float4 w = *reinterpret_cast<const float4*>(row + c);
    x[0] = w.x; x[1] = w.y; x[2] = w.z; x[3] = w.w;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = c + e < F ? row[c + e] : 0.f;
  }
}
__device__ __forceinline__ void load4(const uint16_t* row, int c, int F, float (&x)[4]) {
  if (c + 4 <= F) {
    const uint2 w = *reinterpret_cast<const uint2*>(row + c);
    x[0] = __uint_as_float(w.x << 16); x[1] = __uint_as_float(w.x & 0xffff0000u);
    x[2] = __uint_as_float(w.y << 16); x[3] = __uint_as_float(w.y & 0xffff0000u);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = c + e < F ? __uint_as_float((uint32_t)row[c + e] << 16) : 0.f;
  }
}
__device__ __forceinline__ void store4(float* row, int c, int F, const float (&x)[4]) {
  if (c + 4 <= F) {
    *reinterpret_cast<float4*>(row + c) = make_float4(x[0], x[1], x[2], x[3]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (c + e < F) row[c + e] = x[e];
    }
  }
}
__device__ __forceinline__ void store4(uint16_t* row, int c, int F, const float (&x)[4]) {
  typedef ops::Elem<uint16_t> B;
  if (c + 4 <= F) {
    *reinterpret_cast<uint2*>(row + c) = make_uint2(B::pack2(x[0], x[1]), B::pack2(x[2], x[3]));
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (c + e < F) row[c + e] = B::one(x[e]);
    }
  }
}

typedef float floatx2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void from_codes(uint32_t w, float scale, float (&x)[4]) {
  const floatx2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  x[0] = a.x * scale; x[1] = a.y * scale; x[2] = b.x * scale; x[3] = b.y * scale;
}
// The codes of a block's numbers, four a lane, and their scale; a number that is not finite is held as NaN.
template <bool ROOT>
__device__ __forceinline__ uint32_t to_codes(const float (&x)[4], float* scale) {
  float top = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(x[e]) < __builtin_inff() ? fabsf(x[e]) : 0.f);
  top = wave_max(top);
  const uint32_t u = __float_as_uint(top);
  int k = 0;
  if (u) k = max((int)(u >> 23) - 126 - ((u & 0x7fffffu) <= 0x600000u ? 9 : 8), -126);
  *scale = __uint_as_float((uint32_t)(127 + k) << 23);
  const float inverse = __uint_as_float((uint32_t)(127 - k) << 23);
  float y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    y[e] = x[e] * inverse;
    if (ROOT) y[e] = x[e] > 0.f ? fmaxf(y[e], 0.001953125f) : y[e];
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  uint32_t codes = (uint32_t)w;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (!(fabsf(x[e]) < __builtin_inff())) codes |= 0x7fu << (8 * e);
  }
  return codes;
}

template <class E, bool EIGHT, bool MASTER>
__device__ __forceinline__ void step(const StepArgs& a, const Tensor& t, uint32_t index, const Factors& f) {
#pragma clang fp contract(off)
  constexpr int U = 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t at0 = (int64_t)index * kChunk + wave * (U * kBlock) + lane * 4;
  float p[U][4], g[U][4], m[U][4], v[U][4];
  int64_t row[U];
  int col[U];
  bool in[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t at = at0 + u * kBlock;
    in[u] = at < t.total;
    row[u] = 0;
    col[u] = 0;
    if (in[u] && !t.flat) {
      if (t.total >> 32) row[u] = at / t.pitch;
      else row[u] = (uint32_t)at / (uint32_t)t.pitch;
      col[u] = (int)(at - row[u] * t.pitch);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) p[u][e] = g[u][e] = m[u][e] = v[u][e] = 0.f;
    if (!in[u]) continue;
    const int64_t ip = t.flat ? at : row[u] * t.ldp, ig = t.flat ? at : row[u] * t.ldg, im = t.flat ? at : row[u] * t.ldmaster;
    const int c = col[u], F = t.flat ? 4 : t.F;
    if (MASTER) load4(t.master + im, c, F, p[u]);
    else load4(static_cast<const E*>(t.p) + ip, c, F, p[u]);
    load4(static_cast<const E*>(t.g) + ig, c, F, g[u]);
    if (EIGHT) {
      from_codes(*reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(t.m) + at), t.m_scale[at / kBlock], m[u]);
      from_codes(*reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(t.v) + at), t.v_scale[at / kBlock], v[u]);
    } else {
      load4(static_cast<const float*>(t.m) + at, 0, 4, m[u]);
      load4(static_cast<const float*>(t.v) + at, 0, 4, v[u]);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t at = at0 + u * kBlock;
    if (at0 - lane * 4 + u * kBlock >= t.total) break;      // the whole wave
    const int c = col[u], F = t.flat ? 4 : t.F;
    float root[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool real = in[u] && c + e < F;      // columns behind F have states of zero
      if (EIGHT) v[u][e] = v[u][e] * v[u][e];
      m[u][e] = real ? m[u][e] * a.b1 + g[u][e] * a.a1 : 0.f;
      v[u][e] = real ? v[u][e] * a.b2 + (g[u][e] * g[u][e]) * a.a2 : 0.f;
      root[e] = sqrtf(v[u][e]);
      p[u][e] = p[u][e] - f.lr * ((m[u][e] * f.c1) / (root[e] * f.c2 + a.eps) + t.decay * p[u][e]);
    }
    if (in[u]) {
      if (MASTER) store4(t.master + (t.flat ? at : row[u] * t.ldmaster), c, F, p[u]);
      store4(static_cast<E*>(t.p) + (t.flat ? at : row[u] * t.ldp), c, F, p[u]);
    }
    if (EIGHT) {
      float sm, sv;
      const uint32_t cm = to_codes<false>(m[u], &sm), cv = to_codes<true>(root, &sv);
      if (in[u]) {
        *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(t.m) + at) = cm;
        *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(t.v) + at) = cv;
      }
      if (lane == 0) t.m_scale[at / kBlock] = sm, t.v_scale[at / kBlock] = sv;
    } else if (in[u]) {
      store4(static_cast<float*>(t.m) + at, 0, 4, m[u]);
      store4(static_cast<float*>(t.v) + at, 0, 4, v[u]);
    }
  }
}

template <bool EIGHT>
__global__ __launch_bounds__(256) void k_adamw(StepArgs a) {
  const Chunk c = a.chunks[blockIdx.x];
  const Tensor t = a.tensors[c.tensor];
  const Factors f = a.device ? *a.device : a.host;
  if (t.bf16) {
    if (t.master) step<uint16_t, EIGHT, true>(a, t, c.index, f);
    else step<uint16_t, EIGHT, false>(a, t, c.index, f);
  } else {
    step<float, EIGHT, false>(a, t, c.index, f);
  }
}

// The step's number and learning rate where they live on the device.
__global__ void k_adamw_count(int64_t* steps, const float* lr_at, float lr, double b1, double b2, Factors* to) {
  const int64_t t = *steps + 1;
  *steps = t;
  if (!to) return;      // nothing to step: it counts all the same
  to->lr = lr_at ? *lr_at : lr;
  to->c1 = (float)(1. / (1. - pow(b1, (double)t)));
  to->c2 = (float)(1. / sqrt(1. - pow(b2, (double)t)));
}

int64_t pitch_of(int64_t F) { return (F + 15) / 16 * 16; }

const char* check(const dgc_adamw_tensor_t& t, int32_t bits) {
  if (t.dtype != DGC_DTYPE_F32 && t.dtype != DGC_DTYPE_BF16) return "adamw: unknown dtype";
  if (t.R < 0 || t.F < 0 || t.F > (1 << 30)) return "adamw: R must be >= 0 and F in [0, 2^30]";
  if (t.R == 0 || t.F == 0) return nullptr;
  const int e = ops::elem_bytes(t.dtype);
  if (t.R > ((int64_t)1 << 43) / pitch_of(t.F)) return "adamw: a tensor is too large";
  const int64_t ldp = t.R == 1 ? pitch_of(t.F) : t.ldp, ldg = t.R == 1 ? pitch_of(t.F) : t.ldg, ldm = t.R == 1 ? pitch_of(t.F) : t.ldmaster;
  if (!ops::good_rows(t.p, t.R, t.F, ldp, e) || !ops::good_rows(t.g, t.R, t.F, ldg, e))
    return "adamw: p and g need a 16-byte aligned base and a pitch that is a multiple of 16 bytes";
  if (t.master && (t.dtype == DGC_DTYPE_F32 || !ops::good_rows(t.master, t.R, t.F, ldm, 4))) return "adamw: a master belongs to a bf16 parameter, with rows as they are";
  if (!t.m || !t.v || !ops::aligned16(t.m) || !ops::aligned16(t.v)) return "adamw: m and v need 16-byte alignment";
  if ((bits == 8) != (t.m_scale != nullptr) || (bits == 8) != (t.v_scale != nullptr)) return "adamw: scales belong to states in 8 bits";
  if (((uintptr_t)t.m_scale | (uintptr_t)t.v_scale) & 3) return "adamw: scales need 4-byte alignment";
  if (!(t.weight_decay >= 0.f)) return "adamw: weight_decay must be >= 0";
  return nullptr;
}

struct Bytes {
  uintptr_t at, end;
  int64_t pitch, width;       // of rows: those side by side in one buffer are apart
};
bool meet(const Bytes& x, const Bytes& y) {
  if (x.at >= y.end || y.at >= x.end) return false;
  if (!x.pitch || x.pitch != y.pitch) return true;
  const uint64_t d = x.at >= y.at ? (x.at - y.at) % x.pitch : (x.pitch - (y.at - x.at) % x.pitch) % x.pitch;
  return d < (uint64_t)y.width || d + x.width > (uint64_t)x.pitch;
}
Bytes rows(const void* p, int64_t R, int64_t F, int64_t ld, int e) {
  const int64_t pitch = R > 1 ? ld * e : 0;
  return {(uintptr_t)p, (uintptr_t)p + (R - 1) * pitch + F * e, pitch, F * e};
}
Bytes whole(const void* p, int64_t bytes) { return {(uintptr_t)p, (uintptr_t)p + bytes, 0, bytes}; }

}  // namespace
}  // namespace dgc

using namespace dgc;

extern "C" {

dgc_status_t dgc_adamw_create(const dgc_adamw_tensor_t* tensors, int32_t n, int32_t bits, dgc_adamw_t** out) try {
  if (!out) return ops::refuse(DGC_ERR_INVALID_ARG, "adamw: NULL out");
  *out = nullptr;
  if (n < 0 || (n > 0 && !tensors)) return ops::refuse(DGC_ERR_INVALID_ARG, "adamw: NULL tensors");
  if (bits != 8 && bits != 32) return ops::refuse(DGC_ERR_INVALID_ARG, "adamw: states have 8 or 32 bits");
  std::vector<Tensor> all;
  std::vector<Chunk> chunks;
  std::vector<Bytes> written, read;
  for (int32_t i = 0; i < n; ++i) {
    const dgc_adamw_tensor_t& t = tensors[i];
    if (const char* msg = check(t, bits)) return ops::refuse(DGC_ERR_INVALID_ARG, msg);
    if (t.R == 0 || t.F == 0) continue;
    Tensor d{};
    d.p = t.p; d.g = t.g; d.master = t.master; d.m = t.m; d.v = t.v; d.m_scale = t.m_scale; d.v_scale = t.v_scale;
    d.F = t.F; d.pitch = (int32_t)pitch_of(t.F); d.bf16 = t.dtype == DGC_DTYPE_BF16; d.decay = t.weight_decay;
    d.ldp = t.R == 1 ? d.pitch : t.ldp; d.ldg = t.R == 1 ? d.pitch : t.ldg; d.ldmaster = !t.master ? 0 : t.R == 1 ? d.pitch : t.ldmaster;
    d.total = t.R * d.pitch;
    d.flat = d.F == d.pitch && d.ldp == d.pitch && d.ldg == d.pitch && (!t.master || d.ldmaster == d.pitch);
    const int e = ops::elem_bytes(t.dtype);
    const int64_t state = d.total * bits / 8, scales = (d.total + kBlock - 1) / kBlock * 4;
    written.push_back(rows(t.p, t.R, t.F, d.ldp, e));
    if (t.master) written.push_back(rows(t.master, t.R, t.F, d.ldmaster, 4));
    written.push_back(whole(t.m, state));
    written.push_back(whole(t.v, state));
    if (bits == 8) {
      written.push_back(whole(t.m_scale, scales));
      written.push_back(whole(t.v_scale, scales));
    }
    read.push_back(rows(t.g, t.R, t.F, d.ldg, e));
    const int64_t of = (d.total + kChunk - 1) / kChunk;
    if ((int64_t)chunks.size() + of >= (1 << 24)) return ops::refuse(DGC_ERR_UNSUPPORTED, "adamw: more parameters than a launch takes (2^36)");
    for (int64_t c = 0; c < of; ++c) chunks.push_back({(int32_t)all.size(), (uint32_t)c});
    all.push_back(d);
  }
  // Each number is written once and by one lane: what is written lies apart from all else.  Sorted by their beginnings, only those that reach
  // beyond the next one's can meet.
  std::vector<std::pair<Bytes, bool>> order;
  for (const Bytes& b : written) order.push_back({b, true});
  for (const Bytes& b : read) order.push_back({b, false});
  std::sort(order.begin(), order.end(), [](const auto& x, const auto& y) { return x.first.at < y.first.at; });
  for (size_t i = 0; i < order.size(); ++i) {
    for (size_t j = i + 1; j < order.size() && order[j].first.at < order[i].first.end; ++j) {
      if ((order[i].second || order[j].second) && meet(order[i].first, order[j].first))
        return ops::refuse(DGC_ERR_INVALID_ARG, "adamw: parameters, masters and states lie apart from each other and the gradients");
    }
  }
  const size_t a = sizeof(Factors) + 4 + all.size() * sizeof(Tensor), bytes = a + chunks.size() * sizeof(Chunk);
  static_assert(sizeof(Factors) + 4 == 16 && sizeof(Tensor) % 8 == 0, "tensors follow the factors, chunks the tensors");
  std::vector<char> image(bytes);       // what may throw comes before the handle
  dgc_adamw* h = new (std::nothrow) dgc_adamw;
  if (!h) return ops::refuse(DGC_ERR_OOM, "adamw: out of host memory");
  h->bits = bits;
  h->tensors = (int32_t)all.size();
  h->chunks = (int64_t)chunks.size();
  if (h->chunks > 0) {
    std::memcpy(image.data() + 16, all.data(), all.size() * sizeof(Tensor));
    std::memcpy(image.data() + a, chunks.data(), chunks.size() * sizeof(Chunk));
    hipError_t err = hipGetDevice(&h->device);
    if (err == hipSuccess) err = hipMalloc(&h->memory, bytes);
    if (err == hipSuccess) err = hipMemcpy(h->memory, image.data(), bytes, hipMemcpyHostToDevice);
    if (err != hipSuccess) {
      if (h->memory) (void)hipFree(h->memory);
      delete h;
      (void)hipGetLastError();
      return ops::refuse(err == hipErrorOutOfMemory ? DGC_ERR_OOM : DGC_ERR_DEVICE, hipGetErrorString(err));
    }
  }
  *out = h;
  return DGC_OK;
} catch (const std::bad_alloc&) {
  return ops::refuse(DGC_ERR_OOM, "adamw: out of host memory");
} catch (...) {
  return ops::refuse(DGC_ERR_DEVICE, "adamw: failed");
}

void dgc_adamw_destroy(dgc_adamw_t* h) {
  if (!h) return;
  if (h->memory) (void)hipFree(h->memory);
  delete h;
}

dgc_status_t dgc_adamw_step(dgc_adamw_t* h, double lr, double beta1, double beta2, double eps, int64_t t, int64_t* steps, const float* lr_at,
                            void* stream) {
  if (!h) return ops::refuse(DGC_ERR_INVALID_ARG, "adamw: NULL handle");
  if (!(beta1 >= 0. && beta1 < 1. && beta2 >= 0. && beta2 < 1.) || !(eps >= 0.) || !(lr >= 0.) || std::isinf(lr) || std::isinf(eps))
    return ops::refuse(DGC_ERR_INVALID_ARG, "adamw: betas must be in [0, 1), lr and eps finite and >= 0");
  if (!steps && t < 1) return ops::refuse(DGC_ERR_INVALID_ARG, "adamw: steps are numbered from 1");
  if (lr_at && !steps) return ops::refuse(DGC_ERR_INVALID_ARG, "adamw: lr on the device goes with steps on the device");
  if (((uintptr_t)steps & 7) || ((uintptr_t)lr_at & 3)) return ops::refuse(DGC_ERR_INVALID_ARG, "adamw: steps needs 8-byte and lr 4-byte alignment");
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (h->chunks == 0) {
    if (!steps) return DGC_OK;
    hipLaunchKernelGGL(k_adamw_count, 1, 1, 0, st, steps, lr_at, (float)lr, beta1, beta2, static_cast<Factors*>(nullptr));
    return ops::launched("adamw");
  }
  int device = -1;
  if (hipGetDevice(&device) != hipSuccess || device != h->device) return ops::refuse(DGC_ERR_INVALID_ARG, "adamw: another device is current than the handle's");
  char* const mem = static_cast<char*>(h->memory);
  StepArgs a{};
  a.tensors = reinterpret_cast<const Tensor*>(mem + 16);
  a.chunks = reinterpret_cast<const Chunk*>(mem + 16 + h->tensors * sizeof(Tensor));
  a.b1 = (float)beta1; a.a1 = (float)(1. - beta1); a.b2 = (float)beta2; a.a2 = (float)(1. - beta2); a.eps = (float)eps;
  if (steps) {
    a.device = reinterpret_cast<const Factors*>(mem);
    hipLaunchKernelGGL(k_adamw_count, 1, 1, 0, st, steps, lr_at, (float)lr, beta1, beta2, reinterpret_cast<Factors*>(mem));
  } else {
    a.host = {(float)lr, (float)(1. / (1. - std::pow(beta1, (double)t))), (float)(1. / std::sqrt(1. - std::pow(beta2, (double)t)))};
  }
  if (h->bits == 8) hipLaunchKernelGGL(k_adamw<true>, (unsigned)h->chunks, 256, 0, st, a);
  else hipLaunchKernelGGL(k_adamw<false>, (unsigned)h->chunks, 256, 0, st, a);
  return ops::launched("adamw");
}

}  // extern "C"
