// Softmax attention: the C entries, what they refuse, and workspaces.
#include <algorithm>
#include <cmath>
#include <numeric>

#include "dgc_attn_dev.h"

using namespace dgc;
using namespace dgc::attn;

namespace {

constexpr int64_t kMostBlocks = ((int64_t)1 << 24) - 1;      // of 256 threads: a launch holds fewer than 2^32 threads
constexpr int64_t kMostTokens = (int64_t)1 << 30;

const char* check(int64_t Tq, int64_t Tk, int64_t N, int32_t heads, int32_t kv_heads, int32_t d, int32_t dtype, int32_t buckets, int32_t reach) {
  if (dtype != DGC_DTYPE_F32 && dtype != DGC_DTYPE_BF16) return "attention: unknown dtype";
  if (Tq < 0 || Tk < Tq || Tk > kMostTokens || N < 0) return "attention: needs 0 <= Tq <= Tk <= 2^30 and N >= 0";
  if (heads < 1 || heads > kMaxHeads || kv_heads < 1 || heads % kv_heads) return "attention: heads must be in [1, 1024] and a multiple of kv_heads";
  if (d < 8 || d > kMaxDim || d % 8) return "attention: d must be a multiple of 8 in [8, 128]";
  if (buckets < 0 || buckets > kMaxBuckets || reach < 0 || reach > kMaxReach || (buckets == 0 && reach != 0))
    return "attention: buckets must be in [0, 256] (0: no bias) and reach in [0, 1024]";
  return nullptr;
}
bool too_many(int64_t Tq, int64_t Tk, int64_t N, int32_t heads) {      // workgroups of any of the launches, 64 queries or keys each
  return N > kMostBlocks || N * heads > kMostBlocks / ((Tk + 63) / 64 + 1) || N * heads > INT64_MAX / 16 / (Tk + 1);
}

int64_t round16(int64_t bytes) { return (bytes + 15) / 16 * 16; }

// Parts of the keys of a few queries: enough workgroups to fill the card, of 256 keys at least.
int32_t splits_of(int64_t Tq, int64_t Tk, int64_t N, int32_t heads, int32_t kv_heads) {
  const int64_t rows = heads / kv_heads * Tq, items = std::max<int64_t>(1, N * kv_heads * ((rows + 15) / 16));
  return (int32_t)std::max<int64_t>(1, std::min<int64_t>({(1024 + items - 1) / items, Tk / 256, kMaxSplits}));
}
struct Room {
  int64_t delta, odd, part, joint;      // bytes
};
Room back_room(int64_t Tq, int64_t Tk, int64_t N, int32_t heads, int32_t kv_heads, int32_t d, int32_t dtype, int32_t causal, int32_t buckets, int32_t reach) {
  // `first`, which decides between the two forms, is not known here.
  const bool window = takes_window_back(Tk, d, heads / kv_heads, false);
  // A flag for each workgroup of the kernels that have one, 64 queries or keys each.
  Room r{round16(4 * N * heads * Tq), 0, 0, 0};
  const Parts p = key_parts(Tq, Tk, N, heads, kv_heads, dtype == DGC_DTYPE_F32);
  r.odd = round16(4 * N * std::max<int64_t>(heads * ((Tq + 63) / 64), kv_heads * ((Tk + 63) / 64) * p.heads * p.rows));
  if (p.heads * p.rows > 1) r.joint = 8 * N * kv_heads * Tk * d * p.heads * p.rows;
  if (buckets) {
    // The larger of both row tiles' numbers of blocks.
    r.part = 4 * (int64_t)heads * back_slots(false, N, heads, 0, (Tq + 63) / 64, at_once(dtype == DGC_DTYPE_F32, d)) * table_size(reach, causal);
    if (window) r.part = std::max<int64_t>(r.part, 4 * (int64_t)heads * back_slots(true, N, heads, kv_heads, 0, 0) * 64);
    if (window) {
      const WindowPlan p = plan_windows(N, heads, d, ops::elem_bytes(dtype));
      r.part = std::max<int64_t>(r.part, 4 * (int64_t)heads * p.slots * p.tables * 64);
    }
    r.part = round16(r.part);
  }
  return r;
}

// Inputs may repeat rows (a stride of 0); an output's rows lie apart.
bool good(const Rows& x, int64_t T, int64_t N, int64_t F, int e, bool output) {
  if (T == 0 || N == 0) return true;
  const int64_t per = 16 / e, most = INT64_MAX / 32;
  if (!x.p || !ops::aligned16(x.p) || x.st < 0 || x.sn < 0 || x.st % per || x.sn % per) return false;
  if (x.st > most / T || x.sn > most / N) return false;
  if (!output) return true;
  if (T > 1 && N > 1) return x.st >= x.sn ? x.sn >= F && x.st >= N * x.sn : x.st >= F && x.sn >= T * x.st;
  return T > 1 ? x.st >= F : N > 1 ? x.sn >= F : true;
}
struct Span {
  const void* p;
  int64_t T, N, st, sn, F, e;       // T N rows of F elements of e bytes
  uintptr_t begin() const { return (uintptr_t)p; }
  uintptr_t end() const { return (uintptr_t)p + ((T - 1) * st + (N - 1) * sn + F) * e; }
  bool none() const { return !p || T <= 0 || N <= 0 || F <= 0; }
};
Span of(const Rows& x, int64_t T, int64_t N, int64_t F, int e) { return {x.p, T, N, x.st, x.sn, F, e}; }
Span of(const void* p, int64_t n, int64_t e) { return {p, 1, 1, 0, 0, n, e}; }
// Whether two tensors share a byte.  All their rows start at multiples of the strides' common divisor: rows that do not meet within that do not
// meet, as those side by side in one buffer.
bool meet(const Span& x, const Span& y) {
  if (x.none() || y.none() || x.begin() >= y.end() || y.begin() >= x.end()) return false;
  int64_t g = 0;
  for (const Span* s : {&x, &y}) {
    if (s->T > 1) g = std::gcd(g, s->st * s->e);
    if (s->N > 1) g = std::gcd(g, s->sn * s->e);
  }
  if (g == 0) return true;
  const uint64_t d = x.begin() >= y.begin() ? (x.begin() - y.begin()) % g : (g - (y.begin() - x.begin()) % g) % g;
  return d < (uint64_t)(y.F * y.e) || d + (uint64_t)(x.F * x.e) > (uint64_t)g;
}

constexpr const char* kBadRows = "attention: tensors need a 16-byte aligned base and strides that are multiples of 16 bytes; an output's rows lie apart";
constexpr const char* kMeet = "attention: outputs lie apart from the inputs and each other";
constexpr const char* kWorkspace = "attention: workspace missing, too small (dgc_attn_workspace_bytes) or not 16-byte aligned";

bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }

const char* fill(Args* a, int64_t Tq, int64_t Tk, int64_t N, int32_t heads, int32_t kv_heads, int32_t d, int32_t causal, float scale, const int32_t* first,
                 const int32_t* lengths, const uint8_t* keep, const float* bias, const uint8_t* map, int32_t buckets, int32_t reach) {
  if ((buckets > 0) != (bias != nullptr) || (buckets > 0) != (map != nullptr)) return "attention: bias, bias_map and buckets go together";
  if (!aligned4(first) || !aligned4(lengths) || !aligned4(bias)) return "attention: first, lengths and bias need 4-byte alignment";
  a->N = N; a->Tq = (int32_t)Tq; a->Tk = (int32_t)Tk; a->heads = heads; a->group = heads / kv_heads; a->d = d; a->causal = causal != 0; a->scale = scale;
  a->first = first; a->lengths = lengths; a->keep = keep; a->bias = bias; a->map = map; a->buckets = buckets; a->reach = reach;
  return nullptr;
}

}  // namespace

extern "C" {

dgc_status_t dgc_attn_buckets(int32_t buckets, int32_t reach, int32_t causal, uint8_t* host_out) {
  if (!host_out || buckets < 2 || buckets > kMaxBuckets || (!causal && (buckets % 2 || buckets < 4)) || reach < 1 || reach > kMaxReach)
    return ops::refuse(DGC_ERR_INVALID_ARG, "attention buckets: buckets in [2, 256] (even and at least 4 for both sides), reach in [1, 1024]");
  // Bucket single + k begins at single (reach / single)^(k / (side - single)): in logarithms, with room for their rounding.
  const int side = causal ? buckets : buckets / 2, single = side / 2;
  if (reach < single) return ops::refuse(DGC_ERR_INVALID_ARG, "attention buckets: reach is less than the distances that have a bucket of their own");
  for (int x = 0; x <= reach; ++x) {
    int b = x;
    if (x >= single && single > 0) {
      const double at = reach > single ? std::log((double)x / single) / std::log((double)reach / single) * (side - single) : side - single;
      b = std::min(side - 1, single + (int)(at + 1e-9));
    }
    host_out[reach + x] = (uint8_t)b;
    if (x) host_out[reach - x] = (uint8_t)(causal ? 0 : side + b);
  }
  return DGC_OK;
}

int64_t dgc_attn_workspace_bytes(int64_t Tq, int64_t Tk, int64_t N, int32_t heads, int32_t kv_heads, int32_t d, int32_t dtype, int32_t causal,
                                 int32_t buckets, int32_t reach, int32_t backward) {
  if (check(Tq, Tk, N, heads, kv_heads, d, dtype, buckets, reach) || too_many(Tq, Tk, N, heads)) return -1;
  if (N == 0 || Tk == 0) return 0;
  if (backward) {      // without queries, too: keys have gradients of zero
    const Room r = back_room(Tq, Tk, N, heads, kv_heads, d, dtype, causal, buckets, reach);
    return r.delta + r.odd + r.part + r.joint;
  }
  if (Tq == 0 || form_of(Tq, Tk) != kFew) return 0;
  const int64_t splits = splits_of(Tq, Tk, N, heads, kv_heads);
  return splits > 1 ? round16(4 * N * heads * Tq * splits * (d + 2)) : 0;
}

dgc_status_t dgc_attn_forward(const void* q, int64_t qt, int64_t qn, const void* k, int64_t kt, int64_t kn, const void* v, int64_t vt, int64_t vn,
                              int64_t Tq, int64_t Tk, int64_t N, int32_t heads, int32_t kv_heads, int32_t d, int32_t dtype, int32_t causal, float scale,
                              const int32_t* first, const int32_t* lengths, const uint8_t* keep, const float* bias, const uint8_t* bias_map,
                              int32_t buckets, int32_t reach, void* o, int64_t ot, int64_t on, float* lse, void* workspace, int64_t workspace_bytes,
                              void* stream) {
  if (const char* msg = check(Tq, Tk, N, heads, kv_heads, d, dtype, buckets, reach)) return ops::refuse(DGC_ERR_INVALID_ARG, msg);
  if (too_many(Tq, Tk, N, heads)) return ops::refuse(DGC_ERR_UNSUPPORTED, "attention: more sequences, heads and tokens than a launch takes");
  const int e = ops::elem_bytes(dtype);
  const int64_t fq = (int64_t)heads * d, fk = (int64_t)kv_heads * d;
  Args a{};
  a.q = {q, qt, qn}; a.k = {k, kt, kn}; a.v = {v, vt, vn}; a.o = {o, ot, on};
  if (!good(a.q, Tq, N, fq, e, false) || !good(a.k, Tk, N, fk, e, false) || !good(a.v, Tk, N, fk, e, false) || !good(a.o, Tq, N, fq, e, true))
    return ops::refuse(DGC_ERR_INVALID_ARG, kBadRows);
  if (const char* msg = fill(&a, Tq, Tk, N, heads, kv_heads, d, causal, scale, first, lengths, keep, bias, bias_map, buckets, reach))
    return ops::refuse(DGC_ERR_INVALID_ARG, msg);
  if (!aligned4(lse)) return ops::refuse(DGC_ERR_INVALID_ARG, "attention: lse needs 4-byte alignment");
  const int64_t need = dgc_attn_workspace_bytes(Tq, Tk, N, heads, kv_heads, d, dtype, causal, buckets, reach, 0);
  if (need > 0 && (!workspace || !ops::aligned16(workspace) || workspace_bytes < need)) return ops::refuse(DGC_ERR_INVALID_ARG, kWorkspace);
  const Span in[9] = {of(a.q, Tq, N, fq, e), of(a.k, Tk, N, fk, e), of(a.v, Tk, N, fk, e), of(first, N, 4), of(lengths, N, 4), of(keep, N * Tk, 1),
                      of(bias, (int64_t)heads * buckets, 4), of(bias_map, 2 * (int64_t)reach + 1, 1), of(need > 0 ? workspace : nullptr, need, 1)};
  const Span out[2] = {of(a.o, Tq, N, fq, e), of(lse, N * heads * Tq, 4)};
  for (const Span& x : out) {
    for (const Span& y : in) {
      if (meet(x, y)) return ops::refuse(DGC_ERR_INVALID_ARG, kMeet);
    }
  }
  for (int x = 0; x < 8; ++x) {
    if (meet(in[x], in[8])) return ops::refuse(DGC_ERR_INVALID_ARG, kMeet);
  }
  if (meet(out[0], out[1])) return ops::refuse(DGC_ERR_INVALID_ARG, kMeet);
  if (N == 0 || Tq == 0) return DGC_OK;
  a.lse = lse;
  a.splits = form_of(Tq, Tk) == kFew ? splits_of(Tq, Tk, N, heads, kv_heads) : 1;
  a.joint = static_cast<float*>(workspace);
  (dtype == DGC_DTYPE_F32 ? attn_forward_f32 : attn_forward_bf16)(a, static_cast<hipStream_t>(stream));
  return ops::launched("attention");
}

dgc_status_t dgc_attn_backward(const void* q, int64_t qt, int64_t qn, const void* k, int64_t kt, int64_t kn, const void* v, int64_t vt, int64_t vn,
                               const void* o, int64_t ot, int64_t on, const float* lse, const void* go, int64_t gt, int64_t gn, int64_t Tq, int64_t Tk,
                               int64_t N, int32_t heads, int32_t kv_heads, int32_t d, int32_t dtype, int32_t causal, float scale, const int32_t* first,
                               const int32_t* lengths, const uint8_t* keep, const float* bias, const uint8_t* bias_map, int32_t buckets, int32_t reach,
                               void* dq, int64_t dqt, int64_t dqn, void* dkey, int64_t dkt, int64_t dkn, void* dval, int64_t dvt, int64_t dvn,
                               float* dbias, void* workspace, int64_t workspace_bytes, void* stream) {
  if (const char* msg = check(Tq, Tk, N, heads, kv_heads, d, dtype, buckets, reach)) return ops::refuse(DGC_ERR_INVALID_ARG, msg);
  if (too_many(Tq, Tk, N, heads)) return ops::refuse(DGC_ERR_UNSUPPORTED, "attention: more sequences, heads and tokens than a launch takes");
  const int e = ops::elem_bytes(dtype);
  const int64_t fq = (int64_t)heads * d, fk = (int64_t)kv_heads * d;
  Args a{};
  a.q = {q, qt, qn}; a.k = {k, kt, kn}; a.v = {v, vt, vn}; a.o = {o, ot, on}; a.go = {go, gt, gn};
  a.dq = {dq, dqt, dqn}; a.dk = {dkey, dkt, dkn}; a.dv = {dval, dvt, dvn};
  if (!good(a.q, Tq, N, fq, e, false) || !good(a.k, Tk, N, fk, e, false) || !good(a.v, Tk, N, fk, e, false) || !good(a.o, Tq, N, fq, e, false) ||
      !good(a.go, Tq, N, fq, e, false) || (dq && !good(a.dq, Tq, N, fq, e, true)) || (dkey && !good(a.dk, Tk, N, fk, e, true)) ||
      (dval && !good(a.dv, Tk, N, fk, e, true)))
    return ops::refuse(DGC_ERR_INVALID_ARG, kBadRows);
  if (const char* msg = fill(&a, Tq, Tk, N, heads, kv_heads, d, causal, scale, first, lengths, keep, bias, bias_map, buckets, reach))
    return ops::refuse(DGC_ERR_INVALID_ARG, msg);
  if ((!lse && N * Tq > 0) || !aligned4(lse)) return ops::refuse(DGC_ERR_INVALID_ARG, "attention: lse is NULL or not 4-byte aligned");
  if ((dbias && !buckets) || !aligned4(dbias)) return ops::refuse(DGC_ERR_INVALID_ARG, "attention: dbias without a bias, or not 4-byte aligned");
  const int64_t need = dgc_attn_workspace_bytes(Tq, Tk, N, heads, kv_heads, d, dtype, causal, buckets, reach, 1);
  if (need > 0 && (!workspace || !ops::aligned16(workspace) || workspace_bytes < need)) return ops::refuse(DGC_ERR_INVALID_ARG, kWorkspace);
  const Span in[12] = {of(a.q, Tq, N, fq, e), of(a.k, Tk, N, fk, e), of(a.v, Tk, N, fk, e), of(a.o, Tq, N, fq, e), of(a.go, Tq, N, fq, e), of(lse, N * heads * Tq, 4),
                       of(first, N, 4), of(lengths, N, 4), of(keep, N * Tk, 1), of(bias, (int64_t)heads * buckets, 4), of(bias_map, 2 * (int64_t)reach + 1, 1),
                       of(need > 0 ? workspace : nullptr, need, 1)};
  const Span out[4] = {of(a.dq, Tq, N, fq, e), of(a.dk, Tk, N, fk, e), of(a.dv, Tk, N, fk, e), of(dbias, (int64_t)heads * buckets, 4)};
  for (int x = 0; x < 4; ++x) {
    for (const Span& y : in) {
      if (meet(out[x], y)) return ops::refuse(DGC_ERR_INVALID_ARG, kMeet);
    }
    for (int y = 0; y < x; ++y) {
      if (meet(out[x], out[y])) return ops::refuse(DGC_ERR_INVALID_ARG, kMeet);
    }
  }
  for (int x = 0; x < 11; ++x) {
    if (meet(in[x], in[11])) return ops::refuse(DGC_ERR_INVALID_ARG, kMeet);
  }
  a.lse = const_cast<float*>(lse);
  const Room r = back_room(Tq, Tk, N, heads, kv_heads, d, dtype, causal, buckets, reach);
  a.joint = reinterpret_cast<float*>(static_cast<char*>(workspace) + r.delta + r.odd + r.part);
  a.odd = reinterpret_cast<int32_t*>(static_cast<char*>(workspace) + r.delta);
  a.delta = static_cast<float*>(workspace);
  a.part = dbias && N > 0 && Tq > 0 ? reinterpret_cast<float*>(static_cast<char*>(workspace) + r.delta + r.odd) : nullptr;
  (dtype == DGC_DTYPE_F32 ? attn_backward_f32 : attn_backward_bf16)(a, dbias, static_cast<hipStream_t>(stream));
  return ops::launched("attention");
}

}  // extern "C"
