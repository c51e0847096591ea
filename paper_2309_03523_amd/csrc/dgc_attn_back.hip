// Softmax attention over the tokens of sequences, backward.  With the forward pass' o and lse, for every query i and key j that it sees:
//
//   P = e^(s - lse),  dP = do_i . v_j,  D = do_i . o_i,  dS = P (dP - D)
//   dv_j = sum_i P do_i,  dq_i = scale sum_j dS k_j,  dk_j = scale sum_i dS q_i,  dbias[h][b] = sum of dS over the pairs whose distance has bucket b
//
// Scores are computed again, not kept.  In k_attn_dq queries are columns and keys are summed over, in k_attn_dkv keys are columns and queries are summed over
// (heads that share a key head one after the other), so no two workgroups add to one number: no atomics on memory, one order of sums, at the price of
// seven products for five.  Windows of up to 32 keys have a whole sequence and head in a wave and need five: k_attn_windows_back where every head has a key head of its
// own and the rows fit 64 KB of LDS, k_attn_window_back where up to four share one, or they do not.  The others: k_attn_delta (D), k_attn_dq, k_attn_dkv, k_attn_dkv_join (parts of the queries).
// Rounding: bf16 tensors enter products as they are, scores, P, dP, D and dS are fp32; P and dS are rounded to bf16 (by up to 2^-8 of themselves)
// for the products of dv, dq and dk, which are summed in fp32; the bias' gradient sums dS as it is, in fp32 and at the end in double.
//
// The bias' gradient: every wave sums dS by distance into a table of its own in LDS.  In k_attn_dq it lays a tile's dS out slanted, so that a distance is
// a column, and each lane sums one (adding with LDS atomics took 126 cycles an instruction, five times as much).  In
// k_attn_window_back tiles are few and atomics do: each of the four rows of lanes holds one key and neighbouring queries, whose distances differ, and
// has a table, so an instruction never adds twice to one place.  All sums have one order; k_attn_bias joins the tables.
#include <algorithm>
#include <type_traits>

#include "dgc_attn_dev.h"

namespace dgc {
namespace attn {
namespace {

__device__ __forceinline__ void add_lds(float* to, float x) { __hip_atomic_fetch_add(to, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT); }

// ---------------------------------------------------------------------------------------------------- windows
//
// A wave takes one sequence and key head after the other; keys, queries and their gradients lie in its part of LDS, so no wave waits for another.
template <class Tl, int NT, int KS>
__global__ __launch_bounds__(256) void k_attn_window_back(Args a) {
  typedef typename Tl::E E;
  typedef typename Tl::Frag Frag;
  constexpr int DT = Geometry<Tl, KS>::DT, P = Geometry<Tl, KS>::P, W = 16 * NT, PT = 16 + 16 / (int)sizeof(E);
  __shared__ __attribute__((aligned(16))) E room[4][(W + 32) * P + 2 * 16 * PT];
  extern __shared__ float tables[];       // with a bias: [4 waves][group][1 + 4][2 W], the bias by distance and four tables of sums
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane & 15, sub = lane >> 4, kvs = a.heads / a.group;
  const int64_t id = (int64_t)blockIdx.x * 4 + wave;
  const int y = (int)(id % kvs), slot = (int)(id / kvs);
  if (slot >= a.slots) return;
  E *sk = room[wave], *sq = sk + W * P, *sg = sq + 16 * P, *sp = sg + 16 * P, *ss = sp + 16 * PT;
  float* const mine = tables + wave * a.group * 5 * 2 * W;
  const int at = a.Tk - a.Tq;      // of every first query
  if (a.bias) {
    for (int g = 0; g < a.group; ++g) {
      for (int x = lane; x < 2 * W; x += 64) {
        mine[g * 10 * W + x] = bias_at(a, y * a.group + g, at - W + 1 + x);
        for (int s = 1; s < 5; ++s) mine[g * 10 * W + s * 2 * W + x] = 0.f;
      }
    }
  }
  const auto acc0 = (floatx4)(0.f);
  for (int64_t n = slot; n < a.N; n += a.slots) {
    const int len = a.lengths ? min(max(a.lengths[n], 0), a.Tk) : a.Tk, hi = min(max(len - at, 0), a.Tq);
    const bool there = lane < len && (!a.keep || a.keep[(int64_t)lane * a.N + n]);
    const uint64_t keys = __ballot(there);
    const E* kbase = static_cast<const E*>(a.k.p) + n * a.k.sn + y * a.d;
    const E* vbase = static_cast<const E*>(a.v.p) + n * a.v.sn + y * a.d;
    wave_fence();
    Frag fv[NT][KS];
    bool bad = false;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int j = 16 * t + col;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int c = 16 * s + 4 * sub;
        const bool ok = (keys >> j & 1) && c < a.d;
        const Frag fk = ok ? Tl::load(kbase + j * a.k.st + c) : Tl::zero();
        fv[t][s] = ok ? Tl::load(vbase + j * a.v.st + c) : Tl::zero();
        bad = bad || Tl::odd(fk);
        Tl::store(sk + j * P + c, fk);
      }
    }
    const bool odd_k = a.causal && __any(bad);
    floatx4 dk[NT][DT], dv[NT][DT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) dk[t][dt] = dv[t][dt] = acc0;
    }
    for (int g = 0; g < a.group; ++g) {
      const int h = y * a.group + g;
      float* const table = mine + g * 10 * W;
      const E* qbase = static_cast<const E*>(a.q.p) + n * a.q.sn + h * a.d;
      const E* gbase = static_cast<const E*>(a.go.p) + n * a.go.sn + h * a.d;
      const E* obase = static_cast<const E*>(a.o.p) + n * a.o.sn + h * a.d;
      const float* lses = a.lse + (n * a.heads + h) * a.Tq;
      for (int i0 = 0; i0 < hi; i0 += 16) {
        const int i = i0 + col, p = at + i;
        const float lse = i < hi ? lses[i] : -__builtin_inff();
        const bool live = lse != -__builtin_inff();      // a query that sees nothing has no gradient, and gives none
        const uint64_t sees = !live ? 0 : a.causal && p < 63 ? keys & ((2ull << p) - 1) : keys;
        const int last = a.causal ? at + min(i0 + 16, hi) - 1 : len - 1;
        Frag fq[KS], fg[KS];
        float D = 0.f;
        bool odd_qg = false;
        wave_fence();
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const int c = 16 * s + 4 * sub;
          const bool ok = live && c < a.d;
          fq[s] = ok ? Tl::load(qbase + i * a.q.st + c) : Tl::zero();
          fg[s] = ok ? Tl::load(gbase + i * a.go.st + c) : Tl::zero();
          const Frag fo = ok ? Tl::load(obase + i * a.o.st + c) : Tl::zero();
          D += Tl::dot(fg[s], fo);
          odd_qg = odd_qg || Tl::odd(fq[s]) || Tl::odd(fg[s]);
          Tl::store(sq + col * P + c, fq[s]);
          Tl::store(sg + col * P + c, fg[s]);
        }
        D = column_sum<4>(D);
        odd_qg = a.causal && __any(odd_qg);
        floatx4 dq[DT];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) dq[dt] = acc0;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          if (16 * t > last) break;
          wave_fence();
          floatx4 x = acc0, z = acc0;
#pragma unroll
          for (int s = 0; s < KS; ++s) {
            x = Tl::mma(Tl::rows(sk + 16 * t * P, P, s, lane), fq[s], x);
            z = Tl::mma(fv[t][s], fg[s], z);
          }
          const uint32_t bits = (uint32_t)(sees >> (16 * t + 4 * sub));
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int away = i - (16 * t + 4 * sub + r) + W - 1;
            const bool seen = bits >> r & 1;
            const float v = a.bias ? fmaf(x[r], a.scale, table[away]) : x[r] * a.scale;
            x[r] = seen ? weight_of(v, lse) : 0.f;
            z[r] = seen ? x[r] * (z[r] - D) : 0.f;
            if (a.part) add_lds(table + (1 + sub) * 2 * W + away, z[r]);
          }
          const Frag ds = Tl::pack(z, 0);
          Tl::store(sp + col * PT + 4 * sub, Tl::pack(x, 0));
          Tl::store(ss + col * PT + 4 * sub, ds);
          wave_fence();
          const int apart = 16 * t - at - i0;       // key c is seen from query apart + c of the tile on
          const Packed<Tl> p_t(Tl::across(sp, PT, 0, 0, lane)), ds_t(Tl::across(ss, PT, 0, 0, lane));
          if (!odd_k) gather<Tl, DT>(dq, sk + 16 * t * P, P, Packed<Tl>(ds), lane);
          else gather_seen<Tl, DT>(dq, sk + 16 * t * P, P, Packed<Tl>(ds), lane, [](int) { return 0; }, [&](int c) { return c - apart; });
          if (!odd_qg) {
            gather<Tl, DT>(dv[t], sg, P, p_t, lane);
            gather<Tl, DT>(dk[t], sq, P, ds_t, lane);
          } else {
            auto lo = [&](int c) { return apart + c; };
            auto hi = [](int) { return 15; };
            gather_seen<Tl, DT>(dv[t], sg, P, p_t, lane, lo, hi);
            gather_seen<Tl, DT>(dk[t], sq, P, ds_t, lane, lo, hi);
          }
        }
        if (i < hi && a.dq.p) {
          if (!live) {
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) dq[dt] = acc0;
          }
          store_column<Tl, DT>(static_cast<E*>(const_cast<void*>(a.dq.p)) + i * a.dq.st + n * a.dq.sn + h * a.d, dq, a.scale, a.d, lane);
        }
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int j = 16 * t + col;
      if (j >= len) continue;
      if (!(keys >> j & 1)) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) dk[t][dt] = dv[t][dt] = acc0;
      }
      if (a.dk.p) store_column<Tl, DT>(static_cast<E*>(const_cast<void*>(a.dk.p)) + j * a.dk.st + n * a.dk.sn + y * a.d, dk[t], a.scale, a.d, lane);
      if (a.dv.p) store_column<Tl, DT>(static_cast<E*>(const_cast<void*>(a.dv.p)) + j * a.dv.st + n * a.dv.sn + y * a.d, dv[t], 1.f, a.d, lane);
    }
  }
  if (a.part) {
    wave_fence();
    for (int g = 0; g < a.group; ++g) {
      for (int x = lane; x < 2 * W; x += 64) {
        const float* s = mine + g * 10 * W + x;
        a.part[((int64_t)(y * a.group + g) * a.slots + slot) * 2 * W + x] = (s[2 * W] + s[4 * W]) + (s[6 * W] + s[8 * W]);
      }
    }
  }
}

// The same where every head has a key head of its own, and rows go through LDS as they lie, if they fit 64 KB: bf16 heads of up to 64 (17 to 32 keys: up to 48), fp32 ones of up to
// 32 (17 to 32 keys: 16; 20 000 x 32, 4 heads of 32, fp32: 676 us in the other, 3.9 TB/s; 8 of 64, bf16: 2.33 ms, 2.3 TB/s) (as in the forward pass' k_attn_windows; straight from memory
// they took 1.2 to 1.6 times as long; 20 000 ragged windows of 32, 4 heads of 32, bf16: 0.42 ms, where 0.14 is what a copy of it all takes; it waits for
// LDS and its own chain of products at two waves a SIMD, of 256 registers and some spilled): all gradients take the place of what they are gradients of, and leave from there.  A wave keeps to one head, or two, so
// the bias' gradient is summed in registers, element by element, until the end.
struct WindowBack {
  Args a;
  int32_t together, seqs, groups, pitch, tables;
};
template <class Tl, int NT, int KS, int NC, int HW>      // NC: pieces of 16 bytes of a tensor that a thread takes; HW: heads of a wave
__global__ __launch_bounds__(256, 2) void k_attn_windows_back(WindowBack w) {
  typedef typename Tl::E E;
  typedef typename Tl::Frag Frag;
  const Args& a = w.a;
  constexpr int DT = Geometry<Tl, KS>::DT, W = 16 * NT, PER = 16 / (int)sizeof(E), PT = 16 + PER;
  extern __shared__ __attribute__((aligned(16))) char window_room[];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane & 15, sub = lane >> 4;
  const int group = blockIdx.x % w.groups, slot = blockIdx.x / w.groups, h0 = group * w.together, heads = min(w.together, a.heads - h0), at = a.Tk - a.Tq;
  const int P = w.pitch, rows = w.seqs * W, cpr = heads * a.d / PER;
  E *sk = reinterpret_cast<E*>(window_room), *sv = sk + rows * P, *sq = sv + rows * P, *sg = sq + rows * P, *sp = sg + rows * P + wave * 2 * 16 * PT, *ss = sp + 16 * PT;
  float* add = reinterpret_cast<float*>(sg + rows * P + 4 * 2 * 16 * PT + 64);       // [together][2 W]: the bias by distance
  float* lses = add + w.together * 2 * W;            // [seqs][together][W]
  float* dots = lses + rows * w.together;            // [rows][pieces of a row]: parts of D
  int* there = reinterpret_cast<int*>(dots + rows * (w.together * a.d / PER));      // [seqs][W]: whether a key is there
  int* lens = there + rows;
  for (int x = threadIdx.x; x < 4 * rows * P; x += 256) sk[x] = 0;       // rows behind Tk and Tq meet weights of zero
  for (int x = threadIdx.x; x < heads * 2 * W; x += 256) add[x] = a.bias ? bias_at(a, h0 + x / (2 * W), at + x % (2 * W) - W + 1) : 0.f;
  for (int x = threadIdx.x; x < rows * w.together; x += 256) lses[x] = -__builtin_inff();
  for (int x = threadIdx.x; x < rows; x += 256) there[x] = 0;
  __syncthreads();
  const int kpieces = w.seqs * a.Tk * cpr, qpieces = w.seqs * a.Tq * cpr;
  // A thread's pieces: sequence and row, among the keys' and among the queries' (seqs: none), and column.  Places and distances are made of them each
  // time: kept, they would not fit the registers.
  int kseq[NC], krow[NC], qseq[NC], qrow[NC], px[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int c = threadIdx.x + 256 * i, r = c / cpr;
    px[i] = (c % cpr) * PER;
    kseq[i] = c < kpieces ? r / a.Tk : w.seqs;
    krow[i] = r % a.Tk;
    qseq[i] = c < qpieces ? r / max(a.Tq, 1) : w.seqs;
    qrow[i] = r % max(a.Tq, 1);
  }
  auto place = [&](int seq, int row, int x) { return (seq * W + row) * P + x; };
  auto bytes = [&](const Rows& t, int seq, int row, int x) { return ((uint32_t)seq * (uint32_t)t.sn + (uint32_t)row * (uint32_t)t.st + (uint32_t)x) * (uint32_t)sizeof(E); };
  auto base = [&](const Rows& x, int64_t n0) { return reinterpret_cast<char*>(static_cast<E*>(const_cast<void*>(x.p)) + n0 * x.sn + h0 * a.d); };
  uint4 nk[NC], nv[NC], nq[NC], ng[NC];
  float nl[NC], nd[NC];
  uint32_t nkeep = 0;
  int nlen = 0;
  auto fetch = [&](int64_t n0) __attribute__((always_inline)) {
    const int here = (int)min((int64_t)w.seqs, a.N - n0);
    nkeep = 0;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      bool in = kseq[i] < here;
      if (a.lengths) in = in && krow[i] < a.lengths[n0 + min(kseq[i], here - 1)];
      if (a.keep) in = in && a.keep[krow[i] * a.N + n0 + min(kseq[i], here - 1)];
      nkeep |= in ? 1u << i : 0;
      nk[i] = in ? *reinterpret_cast<const uint4*>(base(a.k, n0) + bytes(a.k, kseq[i], krow[i], px[i])) : make_uint4(0, 0, 0, 0);
      nv[i] = in ? *reinterpret_cast<const uint4*>(base(a.v, n0) + bytes(a.v, kseq[i], krow[i], px[i])) : make_uint4(0, 0, 0, 0);
      bool token = qseq[i] < here;
      if (a.lengths) token = token && at + qrow[i] < a.lengths[n0 + min(qseq[i], here - 1)];
      nq[i] = token ? *reinterpret_cast<const uint4*>(base(a.q, n0) + bytes(a.q, qseq[i], qrow[i], px[i])) : make_uint4(0, 0, 0, 0);
      ng[i] = token ? *reinterpret_cast<const uint4*>(base(a.go, n0) + bytes(a.go, qseq[i], qrow[i], px[i])) : make_uint4(0, 0, 0, 0);
      const uint4 o = token ? *reinterpret_cast<const uint4*>(base(a.o, n0) + bytes(a.o, qseq[i], qrow[i], px[i])) : make_uint4(0, 0, 0, 0);
      nl[i] = token ? a.lse[((n0 + qseq[i]) * a.heads + h0 + px[i] / a.d) * a.Tq + qrow[i]] : -__builtin_inff();
      float x[PER], y[PER];
      ops::Elem<E>::unpack(ng[i], x);
      ops::Elem<E>::unpack(o, y);
      nd[i] = 0.f;
#pragma unroll
      for (int e = 0; e < PER; ++e) nd[i] = fmaf(x[e], y[e], nd[i]);
    }
    if ((int)threadIdx.x < w.seqs) nlen = (int)threadIdx.x >= here ? 0 : a.lengths ? min(max(a.lengths[n0 + threadIdx.x], 0), a.Tk) : a.Tk;
  };
  auto put = [&]() __attribute__((always_inline)) -> bool {
    bool odd = false;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      // A query that sees nothing gives no gradient: its rows are zero, whatever they hold.
      const bool live = nl[i] != -__builtin_inff();
      const uint4 q = kept(nq[i], live), g = kept(ng[i], live);
      if (kseq[i] < w.seqs) {
        *reinterpret_cast<uint4*>(sk + place(kseq[i], krow[i], px[i])) = nk[i];
        *reinterpret_cast<uint4*>(sv + place(kseq[i], krow[i], px[i])) = nv[i];
        if (px[i] == 0) there[kseq[i] * W + krow[i]] = nkeep >> i & 1;
      }
      if (qseq[i] < w.seqs) {
        *reinterpret_cast<uint4*>(sq + place(qseq[i], qrow[i], px[i])) = q;
        *reinterpret_cast<uint4*>(sg + place(qseq[i], qrow[i], px[i])) = g;
        dots[(qseq[i] * W + qrow[i]) * cpr + px[i] / PER] = live ? nd[i] : 0.f;
        if (px[i] % a.d == 0) lses[(qseq[i] * w.together + px[i] / a.d) * W + qrow[i]] = nl[i];
      }
      if constexpr (sizeof(E) == 2) odd = odd || Wide::odd(nk[i]) || Wide::odd(q) || Wide::odd(g);
      else odd = odd || Full::odd(nk[i]) || Full::odd(q) || Full::odd(g);
    }
    return odd;
  };
  floatx4 sums[HW][NT][NT];
#pragma unroll
  for (int k = 0; k < HW; ++k) {
#pragma unroll
    for (int u = 0; u < NT; ++u) {
#pragma unroll
      for (int t = 0; t < NT; ++t) sums[k][u][t] = (floatx4)(0.f);
    }
  }
  const auto acc0 = (floatx4)(0.f);
  auto unit = [&](int seq, int g, int64_t n, bool some_odd, floatx4 (&sum)[NT][NT]) __attribute__((always_inline)) {
    const uint32_t keys = (uint32_t)__ballot(lane < a.Tk && there[seq * W + (lane & (W - 1))]);
    const int len = uniform(lens[seq]), hi = len - at;       // queries that are tokens
    E *uk = sk + seq * W * P + g * a.d, *uv = sv + seq * W * P + g * a.d, *uq = sq + seq * W * P + g * a.d, *ug = sg + seq * W * P + g * a.d;
    const float* table = add + g * 2 * W + W - 1 + col - 4 * sub;
    bool odd_k = false, odd_qg = false;      // of this sequence and head: others keep their bits
    if (some_odd) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const bool in = 16 * s + 4 * sub < a.d;
          odd_k = odd_k || (in && Tl::odd(Tl::rows(uk + t * 16 * P, P, s, lane)));
          odd_qg = odd_qg || (in && (Tl::odd(Tl::rows(uq + t * 16 * P, P, s, lane)) || Tl::odd(Tl::rows(ug + t * 16 * P, P, s, lane))));
        }
      }
      odd_k = __any(odd_k);
      odd_qg = __any(odd_qg);
    }
    floatx4 dk[NT][DT], dv[NT][DT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) dk[t][dt] = dv[t][dt] = acc0;
    }
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      if (16 * u >= a.Tq || 16 * u >= hi) break;
      const int i = 16 * u + col, p = at + i;
      const float lse = i < a.Tq ? lses[(seq * w.together + g) * W + i] : -__builtin_inff();
      const bool live = lse != -__builtin_inff();
      const uint32_t sees = !live ? 0 : a.causal ? keys & ((2u << p) - 1) : keys;
      const int last = a.causal ? min(at + 16 * u + 15, len - 1) : len - 1;
      Frag fq[KS], fg[KS];
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        fq[s] = Tl::rows(uq + u * 16 * P, P, s, lane);
        fg[s] = Tl::rows(ug + u * 16 * P, P, s, lane);
        if (16 * s + 4 * sub >= a.d) fq[s] = fg[s] = Tl::zero();
      }
      float D = 0.f;
      for (int x = sub; x < a.d / PER; x += 4) D += i < a.Tq ? dots[(seq * W + i) * cpr + g * (a.d / PER) + x] : 0.f;
      D = column_sum<4>(D);
      floatx4 dq[DT];
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) dq[dt] = acc0;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        if (16 * t > last) break;
        floatx4 x = acc0, z = acc0;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          Frag fk = Tl::rows(uk + t * 16 * P, P, s, lane), fv = Tl::rows(uv + t * 16 * P, P, s, lane);
          if (16 * s + 4 * sub >= a.d) fk = fv = Tl::zero();
          x = Tl::mma(fk, fq[s], x);
          z = Tl::mma(fv, fg[s], z);
        }
        const uint32_t bits = sees >> (16 * t + 4 * sub);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const bool seen = bits >> r & 1;
          x[r] = seen ? exp2_((fmaf(x[r], a.scale, table[16 * (u - t) - r]) - lse) * kLog2e) : 0.f;
          z[r] = seen ? x[r] * (z[r] - D) : 0.f;
        }
        sum[u][t] += z;
        const Frag ds = Tl::pack(z, 0);
        wave_fence();
        Tl::store(sp + col * PT + 4 * sub, Tl::pack(x, 0));
        Tl::store(ss + col * PT + 4 * sub, ds);
        wave_fence();
        const Packed<Tl> p_t(Tl::across(sp, PT, 0, 0, lane)), ds_t(Tl::across(ss, PT, 0, 0, lane));
        const int apart = 16 * t - at - 16 * u;       // key c is seen from query apart + c of the tile on
        if (!odd_k) gather<Tl, DT>(dq, uk + t * 16 * P, P, Packed<Tl>(ds), lane);
        else gather_seen<Tl, DT>(dq, uk + t * 16 * P, P, Packed<Tl>(ds), lane, [](int) { return 0; }, [&](int c) { return c - apart; });
        if (!odd_qg) {
          gather<Tl, DT>(dv[t], ug + u * 16 * P, P, p_t, lane);
          gather<Tl, DT>(dk[t], uq + u * 16 * P, P, ds_t, lane);
        } else {
          auto lo = [&](int c) { return apart + c; };
          auto up = [](int) { return 15; };
          gather_seen<Tl, DT>(dv[t], ug + u * 16 * P, P, p_t, lane, lo, up);
          gather_seen<Tl, DT>(dk[t], uq + u * 16 * P, P, ds_t, lane, lo, up);
        }
      }
      wave_fence();       // this tile's queries have been read
      if (!live) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) dq[dt] = acc0;
      }
      if (i < a.Tq && i < hi) store_column<Tl, DT>(uq + i * P, dq, a.scale, a.d, lane);
    }
    wave_fence();
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int j = 16 * t + col;
      if (j >= a.Tk) continue;
      if (!(keys >> j & 1)) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) dk[t][dt] = dv[t][dt] = acc0;
      }
      store_column<Tl, DT>(uk + j * P, dk[t], a.scale, a.d, lane);
      store_column<Tl, DT>(uv + j * P, dv[t], 1.f, a.d, lane);
    }
  };
  const int64_t step = (int64_t)a.slots * w.seqs;
  int64_t n0 = (int64_t)slot * w.seqs;
  fetch(n0);
  for (bool begun = false; ; n0 += step, begun = true) {
    // The gradients of the last sequences, from where those of the next ones go.
    wordx4 out[3][NC];
    {
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        out[0][i] = *reinterpret_cast<const wordx4*>(sq + (qseq[i] < w.seqs ? place(qseq[i], qrow[i], px[i]) : 0));
        out[1][i] = *reinterpret_cast<const wordx4*>(sk + (kseq[i] < w.seqs ? place(kseq[i], krow[i], px[i]) : 0));
        out[2][i] = *reinterpret_cast<const wordx4*>(sv + (kseq[i] < w.seqs ? place(kseq[i], krow[i], px[i]) : 0));
      }
    }
    const bool more = n0 < a.N;
    const bool odd = more && put();
    if (begun) {
      const int64_t m = n0 - step;
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        if (a.dq.p && qseq[i] < w.seqs && at + qrow[i] < lens[qseq[i]]) *reinterpret_cast<wordx4*>(base(a.dq, m) + bytes(a.dq, qseq[i], qrow[i], px[i])) = out[0][i];
        if (kseq[i] < w.seqs && krow[i] < lens[kseq[i]]) {
          if (a.dk.p) *reinterpret_cast<wordx4*>(base(a.dk, m) + bytes(a.dk, kseq[i], krow[i], px[i])) = out[1][i];
          if (a.dv.p) *reinterpret_cast<wordx4*>(base(a.dv, m) + bytes(a.dv, kseq[i], krow[i], px[i])) = out[2][i];
        }
      }
    }
    if (!more) break;
    bool some_odd = false;
    if (a.causal) some_odd = __syncthreads_or(odd);
    else __syncthreads();
    if ((int)threadIdx.x < w.seqs) lens[threadIdx.x] = nlen;
    if (n0 + step < a.N) fetch(n0 + step);
    __syncthreads();       // the lengths
#pragma unroll
    for (int k = 0; k < HW; ++k) {
      const int x = wave + 4 * k, seq = x / w.together, g = x % w.together;
      if (g < heads && n0 + seq < a.N) unit(seq, g, n0 + seq, some_odd, sums[k]);
    }
    __syncthreads();
  }
  if (a.part) {
    // By distance: a wave's sums as a slanted table in its part of the room, a column a lane.
    float* slant = reinterpret_cast<float*>(window_room) + wave * W * 2 * W;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < HW; ++k) {
      const int x = wave + 4 * k, g = x % w.together;
      wave_fence();
#pragma unroll
      for (int u = 0; u < NT; ++u) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int i = 16 * u + col, j = 16 * t + 4 * sub + r;
            slant[i * 2 * W + W - 1 + i - j] = sums[k][u][t][r];
          }
        }
      }
      wave_fence();
      if (g < heads && lane < 2 * W) {
        float s = 0.f;
        for (int i = 0; i < W; ++i) s += (unsigned)(lane - i) < (unsigned)W ? slant[i * 2 * W + lane] : 0.f;
        a.part[((int64_t)(h0 + g) * a.slots * w.tables + slot * w.tables + x / w.together % w.tables) * 2 * W + lane] = s;
      }
    }
  }
}

// ---------------------------------------------------------------------------------------------------- D = do . o, a row of LPR lanes
template <class E, int LPR>
__global__ __launch_bounds__(256) void k_attn_delta(Args a) {
  constexpr int PER = ops::Elem<E>::kPer;
  const int c = (threadIdx.x % LPR) * PER;
  const int64_t rows = (int64_t)a.Tq * a.N * a.heads;
  for (int64_t x = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LPR; x < rows; x += (int64_t)gridDim.x * 256 / LPR) {
    const int h = (int)(x % a.heads);
    const int64_t n = x / a.heads % a.N;
    const int i = (int)(x / a.heads / a.N);
    const Seq q(a, n);
    const bool live = i >= q.lo && i < q.hi;
    float s = 0.f;
    if (live && c < a.d) {
      float g[PER], o[PER];
      ops::Elem<E>::unpack(*reinterpret_cast<const uint4*>(static_cast<const E*>(a.go.p) + (int64_t)i * a.go.st + n * a.go.sn + h * a.d + c), g);
      ops::Elem<E>::unpack(*reinterpret_cast<const uint4*>(static_cast<const E*>(a.o.p) + (int64_t)i * a.o.st + n * a.o.sn + h * a.d + c), o);
#pragma unroll
      for (int e = 0; e < PER; ++e) s = fmaf(g[e], o[e], s);
    }
#pragma unroll
    for (int m = 1; m < LPR; m *= 2) s += __shfl_xor(s, m);
    if (live && c == 0) a.delta[(n * a.heads + h) * a.Tq + i] = s;
  }
}

// ---------------------------------------------------------------------------------------------------- dq, and the bias' gradient
//
// Four sequences of 4096, 8 heads of 64 on 2 key heads, bf16: 0.174 ms, and k_attn_dkv 0.23 (0.19 and 0.25 in a card's first passes).  Both are bound by how long a wave's chain LDS, products, powers, products
// takes with two waves a SIMD.  As the forward pass: 4 M queries a workgroup, keys in tiles of 2 M through LDS.  The product that forms dP starts from -D, so it
// leaves dP - D; in bf16 D is subtracted behind it: that unit cuts sums off, always to one side, and what it leaves of -D is summed up by the bias' gradient, where
// millions of dS nearly cancel (4000 x 200 tokens, 4 heads of 32: off by 5.5e-6 of its norm, now 5e-7).  It costs 2 to 4 % of this kernel, and leaves registers to heads above
// 64 (2 x 4096, 8 heads of 128: 62 spilled and 640 us for all gradients, 41 and 603 us now).
// Where a zero gradient would meet a key that is not finite, this kernel leaves dq to the same one with SEEN, which is launched behind it and takes
// such items alone: with both in one kernel the registers do not do.
template <class Tl, int KS, bool SEEN>
__global__ __launch_bounds__(256, 2) void k_attn_dq(Args a) {
  typedef typename Tl::E E;
  constexpr int M = Tl::M, NT = Geometry<Tl, KS>::NT, kKeys = NT * M, DT = Geometry<Tl, KS>::DT, P = Geometry<Tl, KS>::P;
  __shared__ __attribute__((aligned(16))) E room[2][2 * kKeys * P];
  __shared__ float seens[2][kKeys];
  extern __shared__ float table[];          // the bias by distance, then the waves' tables of sums and their slanted tiles
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = Tl::col(lane), sub = Tl::sub(lane);
  const int blocks = (a.Tq + 4 * M - 1) / (4 * M), h = blockIdx.x % a.heads, slot = blockIdx.x / a.heads, y = h / a.group;
  const int64_t items = a.N * blocks;
  if (SEEN) {
    bool any = false;
    for (int64_t x = slot; x < (items + a.slots - 1) / a.slots * a.slots; x += a.slots) {
      const int64_t item = x / a.slots & 1 ? x / a.slots * a.slots + a.slots - 1 - slot : x;
      any = any || (item < items && a.odd[item * a.heads + h]);
    }
    if (!any) return;
  }
  const BiasTable bt(a);
  const int tfrom = table_from(a.reach, a.causal), tsize = table_size(a.reach, a.causal);
  float* const sums = table + bt.size;
  if (a.bias) {
    bt.fill(a, table, h, true);
    if (!SEEN && a.part) {
      for (int x = threadIdx.x; x < 4 * tsize; x += 256) sums[x] = 0.f;
    }
  }
  float* const mysums = sums + wave * tsize;
  float* const slant = sums + 4 * tsize + wave * (2 * M * M);      // row q: dS of query q at column M - 1 + q - key
  float farsum = 0.f, aheadsum = 0.f;       // sums of tiles that are far off as a whole
  Stage<E, kKeys, KS> nk, nv;
  nk.init(a.k.st, a.d);
  nv.init(a.v.st, a.d);
  for (int64_t round = 0; round * a.slots < items; ++round) {
    // The longest walks first, every second round backwards: with several items a workgroup, long ones go with short ones.
    const int64_t item = round * a.slots + (round & 1 ? a.slots - 1 - slot : slot);
    if (item >= items) continue;
    const int64_t n = item % a.N;
    const int i0 = (int)(blocks - 1 - item / a.N) * 4 * M;
    const Seq q(a, n);
    if (SEEN ? !a.odd[item * a.heads + h] : i0 >= q.hi || i0 + 4 * M <= q.lo) {
      if (!SEEN && threadIdx.x == 0 && a.causal) a.odd[item * a.heads + h] = 0;
      continue;
    }
    const int least = max(i0, q.lo), most = min(i0 + 4 * M, q.hi) - 1;
    const int kend = a.causal ? (int)min((int64_t)q.len, q.at + most + 1) : q.len;
    const int mine = i0 + wave * M, i = mine + col;
    const bool row = i >= q.lo && i < q.hi;
    const int64_t stat = (n * a.heads + h) * a.Tq + i;
    const float given = row ? a.lse[stat] : -__builtin_inff();
    const bool live = given != -__builtin_inff();
    const float lse = live ? given : __builtin_inff();       // of a query without gradients: all weights are zero
    const bool clean = !SEEN && !Tl::kExact && !__any(row && (!live || far_off(lse)));
    const bool some = max(mine, q.lo) < min(mine + M, q.hi);
    const int p0 = some ? (int)(q.at + max(mine, q.lo)) : -1, p1 = some ? (int)(q.at + min(mine + M, q.hi) - 1) : -1, p = live ? (int)(q.at + i) : -1;
    const float* const mytable = table + (a.reach + kPast) - (live ? p : p0) + 4 * sub;      // plus a key's place
    typename Tl::Frag fq[KS], fg[KS];
    const float minus_D = live ? -a.delta[stat] : 0.f;
    constexpr bool behind_D = !SEEN && !Tl::kExact;      // a branch on a.part instead led the compiler to copy dq behind the loop 5 instructions after the product that forms it, of 11 to wait for
    {
      const E* qrow = static_cast<const E*>(a.q.p) + (int64_t)i * a.q.st + n * a.q.sn + h * a.d;
      const E* grow = static_cast<const E*>(a.go.p) + (int64_t)i * a.go.st + n * a.go.sn + h * a.d;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int c = 16 * s + Tl::KE * sub;
        const bool ok = live && c < a.d;
        fq[s] = ok ? *reinterpret_cast<const typename Tl::Frag*>(qrow + c) : Tl::zero();
        fg[s] = ok ? *reinterpret_cast<const typename Tl::Frag*>(grow + c) : Tl::zero();
      }
    }
    const E* kbase = static_cast<const E*>(a.k.p) + n * a.k.sn + y * a.d;
    const E* vbase = static_cast<const E*>(a.v.p) + n * a.v.sn + y * a.d;
    auto there = [&](int j) { return j < kend && (!a.keep || a.keep[(int64_t)j * a.N + n]); };
    // As in the forward pass: where tiles change their kind.
    const int whole = a.keep ? 0 : kend, inside = a.causal ? (int)(q.at + least) + 1 : kend + kKeys;
    int plain_to = !clean ? 0 : min(whole, min(a.causal ? p0 + 1 : kend, a.bias ? p0 - a.reach + 1 : kend));
    int plain_from = !clean || a.causal ? 0x7fffffff : p1 + a.reach;
    const int last = !some ? -1 : a.causal ? p1 : kend;
    auto holes = [&](int j0) { return j0 + kKeys > whole; };
    const bool near = nk.near && nv.near;
    const E *knext = kbase, *vnext = vbase;
    auto fetch = [&](int j0) __attribute__((always_inline)) {
      if (!holes(j0) && near) {
        nk.fetch_all(knext);
        nv.fetch_all(vnext);
        knext += kKeys * a.k.st;
        vnext += kKeys * a.v.st;
      } else {
        nk.fetch(kbase, a.k.st, j0, there);
        nv.fetch(vbase, a.v.st, j0, there);
      }
    };
    // Lays out a tile; whether a zero gradient would meet a key of it that is not finite.
    auto put = [&](int j0, int b) __attribute__((always_inline)) -> bool {
      nk.put(room[b], P);
      nv.put(room[b] + kKeys * P, P);
      if (holes(j0) && threadIdx.x < kKeys) seens[b][threadIdx.x] = there(j0 + (int)threadIdx.x) ? 1.f : 0.f;
      if (j0 + kKeys > inside) return __syncthreads_or(nk.template odd<Tl>());
      __syncthreads();
      return false;
    };
    typename Tl::Acc dq[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) dq[dt] = (typename Tl::Acc)(0.f);

    // One tile.  PLAIN: every query sees all of it, with one bias.  odd: dq is left out, or (SEEN) keys that are not finite reach only those that see them.
    float bias_behind = 0.f, bias_ahead = 0.f;
    auto tile = [&](auto plain, int j0, int buf, bool odd) __attribute__((always_inline)) {
      constexpr bool PLAIN = decltype(plain)::value;
      const E *sk = room[buf], *sv = sk + kKeys * P;
      const bool behind = p0 - (j0 + kKeys - 1) >= a.reach, ahead = p1 - j0 <= -a.reach;
      const float one = behind ? bias_behind : bias_ahead;
      const float mult = a.scale * kLog2e, add = (one - lse) * kLog2e;
#pragma unroll KS >= 3 || SEEN ? 1 : 2
      for (int t = 0; t < NT; ++t) {
        const int first = j0 + t * M;
        if (!PLAIN && (first >= kend || (a.causal && first > p1))) break;
        typename Tl::Acc x = (typename Tl::Acc)(0.f), z = (typename Tl::Acc)(behind_D ? 0.f : minus_D);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          x = Tl::mma(Tl::rows(sk + t * M * P, P, s, lane), fq[s], x);
          z = Tl::mma(Tl::rows(sv + t * M * P, P, s, lane), fg[s], z);
        }
        if (behind_D) {
#pragma unroll
          for (int r = 0; r < Tl::NR; ++r) z[r] += minus_D;
        }
        if (PLAIN) {
#pragma unroll
          for (int r = 0; r < Tl::NR; ++r) z[r] *= exp2_(fmaf(x[r], mult, add));
        } else {
          if (!a.bias || behind || ahead) {
#pragma unroll
            for (int r = 0; r < Tl::NR; ++r) x[r] = fmaf(x[r], a.scale, one);
          } else {
#pragma unroll
            for (int r = 0; r < Tl::NR; ++r) x[r] = fmaf(x[r], a.scale, mytable[first + Tl::row(r)]);
          }
          const bool masked = holes(j0);
          const float* seen = seens[buf] + t * M + 4 * sub;
          const int upto = !live ? -1 : a.causal ? p - first - 4 * sub : M;
#pragma unroll
          for (int r = 0; r < Tl::NR; ++r) {
            const bool out = Tl::row(r) > upto || (masked && seen[Tl::row(r)] == 0.f);
            z[r] = out ? 0.f : z[r] * exp2_((x[r] - lse) * kLog2e);
          }
        }
        if (!SEEN && a.part) {
          if (behind || ahead) {
            float s = 0.f;
#pragma unroll
            for (int r = 0; r < Tl::NR; ++r) s += z[r];
            if (PLAIN && !live) s = 0.f;       // of a row that only fills the tile up: its zeros times a key that is not finite are NaN
            if (behind) farsum += s;
            else aheadsum += s;
          } else {
            float* const at = slant + col * (2 * M + 1) + M - 1 - 4 * sub;
            wave_fence();
#pragma unroll
            for (int r = 0; r < Tl::NR; ++r) at[-Tl::row(r)] = z[r];
            wave_fence();
            if (lane < 2 * M) {
              float s = 0.f;
#pragma unroll 8
              for (int x = 0; x < M; ++x) s += (unsigned)(lane - x) < (unsigned)M ? slant[x * 2 * M + lane] : 0.f;
              const int64_t place = q.at + mine - first + lane - (M - 1) - tfrom;
              if (s != 0.f && place >= 0 && place < tsize) mysums[place] += s;
            }
          }
        }
        if (SEEN && odd) gather_seen<Tl, DT>(dq, sk + t * M * P, P, Packed<Tl>(z), lane, [](int) { return 0; }, [&](int c) { return (int)(q.at + mine + c) - first; });
        else gather<Tl, DT>(dq, sk + t * M * P, P, Packed<Tl>(z), lane);
      }
    };
    fetch(0);
    bool odd = put(0, 0), odds = odd;
    if (a.bias) {
      bias_behind = table[0];
      bias_ahead = table[bt.size - 1];
      if (far_off(bias_behind)) plain_to = 0;
      if (far_off(bias_ahead)) plain_from = 0x7fffffff;
    }
    for (int j0 = 0, buf = 0; j0 < kend; j0 += kKeys, buf ^= 1) {
      const bool next = j0 + kKeys < kend;
      if (next) fetch(j0 + kKeys);
      if (j0 <= last) {
        if (!SEEN && (j0 + kKeys <= plain_to || (j0 >= plain_from && j0 + kKeys <= whole))) tile(std::true_type(), j0, buf, false);
        else tile(std::false_type(), j0, buf, odd);
      }
      if (next) odd = put(j0 + kKeys, buf ^ 1), odds |= odd;
    }
    if (!SEEN && threadIdx.x == 0 && a.causal) a.odd[item * a.heads + h] = odds;
    if (row && a.dq.p && (SEEN || !odds)) {
      if (!live) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) dq[dt] = (typename Tl::Acc)(0.f);
      }
      store_column<Tl, DT>(static_cast<E*>(const_cast<void*>(a.dq.p)) + (int64_t)i * a.dq.st + n * a.dq.sn + h * a.d, dq, a.scale, a.d, lane);
    }
    __syncthreads();      // before the next item's keys
  }
  if (!SEEN && a.part) {
    __syncthreads();
    farsum = wave_sum(farsum);
    aheadsum = wave_sum(aheadsum);
    if (lane == 0) {
      mysums[a.reach - tfrom] += farsum;
      if (!a.causal) mysums[-a.reach - tfrom] += aheadsum;
    }
    __syncthreads();
    for (int x = threadIdx.x; x < tsize; x += 256) {
      float s = 0.f;
      for (int w = 0; w < 4; ++w) s += sums[w * tsize + x];
      a.part[((int64_t)h * a.slots + slot) * tsize + x] = s;
    }
  }
}

// ---------------------------------------------------------------------------------------------------- dk, dv

// Whether a lane's part of a key or value is not finite: its sum of zero times each number tells.
template <class Tl, int KS>
__device__ __forceinline__ bool odd_rows(const typename Tl::Frag (&a)[KS], const typename Tl::Frag (&b)[KS]) {
  float sum = 0.f;
  auto add = [&](uint32_t w) __attribute__((always_inline)) {
    if constexpr (sizeof(typename Tl::E) == 2) sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), bf16x2{0, 0}, sum, false);
    else sum = fmaf(__uint_as_float(w), 0.f, sum);
  };
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    add(a[s].x), add(a[s].y), add(a[s].z), add(a[s].w);
    add(b[s].x), add(b[s].y), add(b[s].z), add(b[s].w);
  }
  return sum != sum;
}

//
// A workgroup takes 4 M keys of one sequence and key head, a wave M of them in registers, and walks over the queries that see them in tiles of
// 2 M that lie in LDS, for one head that shares the keys after the other.  The products that form scores and dP start from -lse / scale and -D of
// their rows, which come from LDS as four numbers at a time: they leave (s - lse) / scale and dP - D.
// Queries that are not finite: as in k_attn_dq.
template <class Tl, int KS, bool SEEN>
__global__ __launch_bounds__(256, KS * Tl::M > 128 ? 1 : SEEN && Tl::M == 32 && KS <= 2 ? 3 : 2) void k_attn_dkv(Args a) {
  typedef typename Tl::E E;
  constexpr int M = Tl::M, NT = M == 32 && KS >= 4 ? 1 : 2, kRows = NT * M, DT = Geometry<Tl, KS>::DT, P = Geometry<Tl, KS>::P;
  __shared__ __attribute__((aligned(16))) E room[2][2 * kRows * P];
  __shared__ __attribute__((aligned(16))) float stats[2][3][kRows];      // lse, -lse / scale, -D
  extern __shared__ float table[];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = Tl::col(lane), sub = Tl::sub(lane), kvs = a.heads / a.group;
  const uint32_t pairs = (uint32_t)(a.N * kvs), pair = blockIdx.x % pairs, rest = blockIdx.x / pairs, parts = a.head_parts * a.row_parts;
  const int64_t n = pair / kvs;
  const int y = pair % kvs, k0 = (int)(rest / parts) * 4 * M, part = rest % parts, head_part = part / a.row_parts, row_part = part % a.row_parts;
  const Seq q(a, n);
  if (SEEN ? !a.odd[blockIdx.x] : k0 >= q.len) {
    if (!SEEN && threadIdx.x == 0 && a.causal) a.odd[blockIdx.x] = 0;
    return;
  }
  const int mine = k0 + wave * M, j = mine + col;
  // A key behind every query counts as masked, whatever it holds.
  const bool there = j < q.len && (!a.causal || j < q.at + q.hi) && (!a.keep || a.keep[(int64_t)j * a.N + n]);
  const BiasTable bt(a);
  const float* const mytable = table - j - bt.from + 4 * sub;      // plus a query's position
  typename Tl::Frag fk[KS], fv[KS];
  {
    const E* krow = static_cast<const E*>(a.k.p) + (int64_t)j * a.k.st + n * a.k.sn + y * a.d;
    const E* vrow = static_cast<const E*>(a.v.p) + (int64_t)j * a.v.st + n * a.v.sn + y * a.d;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int c = 16 * s + Tl::KE * sub;
      const bool ok = there && c < a.d;
      fk[s] = ok ? *reinterpret_cast<const typename Tl::Frag*>(krow + c) : Tl::zero();
      fv[s] = ok ? *reinterpret_cast<const typename Tl::Frag*>(vrow + c) : Tl::zero();
    }
  }
  typename Tl::Acc dk[DT], dv[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) dk[dt] = dv[dt] = (typename Tl::Acc)(0.f);
  const int begin_all = a.causal ? (int)min((int64_t)q.hi, max((int64_t)q.lo, k0 - q.at)) : q.lo;      // the first query that sees one of these keys
  Stage<E, kRows, KS> nq, ng;
  nq.init(a.q.st, a.d);
  ng.init(a.go.st, a.d);
  const bool near = nq.near && ng.near;
  constexpr int NS = Stage<E, kRows, KS>::N;
  const bool started = !SEEN && !Tl::kExact && a.scale > 1e-6f;      // products may start from -lse / scale
  // This workgroup's part of the heads that share the keys, and of their queries.
  const int heads_each = a.group / a.head_parts, rows_each = ((q.hi - begin_all + a.row_parts - 1) / a.row_parts + kRows - 1) / kRows * kRows;
  const int begin = min(begin_all + row_part * rows_each, q.hi), end = min(begin + rows_each, q.hi);
  bool odds = false;
  for (int g = head_part * heads_each; g < (head_part + 1) * heads_each; ++g) {
    const int h = y * a.group + g;
    __syncthreads();
    if (a.bias) bt.fill(a, table, h, false);
    const E* qbase = static_cast<const E*>(a.q.p) + n * a.q.sn + h * a.d;
    const E* gbase = static_cast<const E*>(a.go.p) + n * a.go.sn + h * a.d;
    const float* lses = a.lse + (n * a.heads + h) * a.Tq;
    const float* Ds = a.delta + (n * a.heads + h) * a.Tq;
    float nlse = 0.f, nD = 0.f, rowlse[NS];
    auto token = [&](int i) { return i >= q.lo && i < end; };
    auto fetch = [&](int i0) __attribute__((always_inline)) {
      if (i0 + kRows <= end && near) {
        nq.fetch_all(qbase + i0 * a.q.st);
        ng.fetch_all(gbase + i0 * a.go.st);
#pragma unroll
        for (int x = 0; x < NS; ++x) rowlse[x] = nq.has[x] ? lses[i0 + nq.row(x)] : 0.f;
      } else {
        nq.fetch(qbase, a.q.st, i0, token);
        ng.fetch(gbase, a.go.st, i0, token);
#pragma unroll
        for (int x = 0; x < NS; ++x) rowlse[x] = nq.has[x] && token(i0 + nq.row(x)) ? lses[i0 + nq.row(x)] : 0.f;
      }
      if (threadIdx.x < kRows) {
        const int i = i0 + threadIdx.x;
        const float given = token(i) ? lses[i] : -__builtin_inff();
        const bool ok = given != -__builtin_inff();
        nlse = ok ? given : __builtin_inff();      // its weights are zero
        nD = ok ? Ds[i] : 0.f;
      }
    };
    auto put = [&](int i0, int b) __attribute__((always_inline)) -> bool {
      // A query that sees nothing gives no gradient: its rows are zero, whatever they hold.
#pragma unroll
      for (int x = 0; x < NS; ++x) {
        if (__any(rowlse[x] == -__builtin_inff())) {
          if (rowlse[x] == -__builtin_inff()) nq.w[x] = ng.w[x] = make_uint4(0, 0, 0, 0);
        }
      }
      nq.put(room[b], P);
      ng.put(room[b] + kRows * P, P);
      if (threadIdx.x < kRows) {
        stats[b][0][threadIdx.x] = nlse;
        stats[b][1][threadIdx.x] = started ? -nlse / a.scale : 0.f;
        stats[b][2][threadIdx.x] = -nD;
      }
      if (a.causal && q.at + i0 < k0 + 4 * M - 1) return __syncthreads_or(nq.template odd<Tl>() || ng.template odd<Tl>());
      __syncthreads();
      return false;
    };
    // One tile.  PLAIN: all its queries see all of the wave's keys, with one bias.
    float bias_behind = 0.f, bias_ahead = 0.f;
    auto tile = [&](auto plain, int i0, int buf, bool exact, bool odd, bool dead) __attribute__((always_inline)) {
      constexpr bool PLAIN = decltype(plain)::value;
      const E *sq = room[buf], *sg = sq + kRows * P;
      const int first_p = (int)(q.at + i0);
      const bool behind = first_p - (mine + M - 1) >= a.reach, ahead = first_p + kRows - 1 - mine <= -a.reach;
      const float one = behind ? bias_behind : bias_ahead, mult = a.scale * kLog2e, add = one * kLog2e;
#pragma unroll KS >= 3 || SEEN ? 1 : 2
      for (int t = 0; t < NT; ++t) {
        const int pt = first_p + t * M;
        if (!PLAIN && ((a.causal && pt + M - 1 < mine) || i0 + t * M >= end)) continue;
        typename Tl::Acc x, z;
#pragma unroll
        for (int r = 0; r < Tl::NR; r += 4) {
          const float4 u = *reinterpret_cast<const float4*>(stats[buf][2] + t * M + 4 * sub + Tl::row(r));
          z[r] = u.x; z[r + 1] = u.y; z[r + 2] = u.z; z[r + 3] = u.w;
        }
        if (PLAIN || !exact) {
#pragma unroll
          for (int r = 0; r < Tl::NR; r += 4) {
            const float4 u = *reinterpret_cast<const float4*>(stats[buf][1] + t * M + 4 * sub + Tl::row(r));
            x[r] = u.x; x[r + 1] = u.y; x[r + 2] = u.z; x[r + 3] = u.w;
          }
        } else {
          x = (typename Tl::Acc)(0.f);
        }
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          x = Tl::mma(Tl::rows(sq + t * M * P, P, s, lane), fk[s], x);
          z = Tl::mma(Tl::rows(sg + t * M * P, P, s, lane), fv[s], z);
        }
        if (PLAIN) {
#pragma unroll
          for (int r = 0; r < Tl::NR; ++r) {
            x[r] = exp2_(fmaf(x[r], mult, add));
            z[r] *= x[r];
          }
        } else {
          if (!a.bias || behind || ahead) {
#pragma unroll
            for (int r = 0; r < Tl::NR; ++r) x[r] = fmaf(x[r], a.scale, one);
          } else {
#pragma unroll
            for (int r = 0; r < Tl::NR; ++r) x[r] = fmaf(x[r], a.scale, mytable[pt + Tl::row(r)]);
          }
          if (exact) {
#pragma unroll
            for (int r = 0; r < Tl::NR; r += 4) {
              const float4 u = *reinterpret_cast<const float4*>(stats[buf][0] + t * M + 4 * sub + Tl::row(r));
              x[r] -= u.x; x[r + 1] -= u.y; x[r + 2] -= u.z; x[r + 3] -= u.w;
            }
            if (dead) {
#pragma unroll
              for (int r = 0; r < Tl::NR; ++r) {
                const bool none = stats[buf][0][t * M + 4 * sub + Tl::row(r)] == __builtin_inff();
                x[r] = none ? -__builtin_inff() : x[r];
                z[r] = none ? 0.f : z[r];
              }
            }
          }
          const int least = a.causal ? j - pt - 4 * sub : -1;
#pragma unroll
          for (int r = 0; r < Tl::NR; ++r) {
            const bool out = Tl::row(r) < least;
            x[r] = out ? 0.f : exp2_(x[r] * kLog2e);
            z[r] = out ? 0.f : z[r] * x[r];
          }
        }
        if (SEEN && odd) {
          auto lo = [&](int c) { return mine + c - pt; };
          auto hi = [](int) { return M - 1; };
          gather_seen<Tl, DT>(dv, sg + t * M * P, P, Packed<Tl>(x), lane, lo, hi);
          gather_seen<Tl, DT>(dk, sq + t * M * P, P, Packed<Tl>(z), lane, lo, hi);
        } else {
          gather<Tl, DT>(dv, sg + t * M * P, P, Packed<Tl>(x), lane);
          gather<Tl, DT>(dk, sq + t * M * P, P, Packed<Tl>(z), lane);
        }
      }
    };
    if (begin >= end) continue;
    // This wave: its keys are seen from query `from_i` on, and by all of a tile from `full_i` on; `plain_from`, `plain_to`: with one bias, behind or ahead.
    const int from_i = mine >= q.len ? 0x7fffffff : a.causal ? (int)(mine - q.at) - (kRows - 1) : begin;
    int plain_from = !started ? 0x7fffffff : (int)min(max(a.causal ? mine + M - 1 - q.at : (int64_t)begin, a.bias ? mine + M - 1 + a.reach - q.at : (int64_t)begin), (int64_t)0x7fffffff);
    int plain_to = !started || a.causal || !a.bias ? -1 : (int)max(mine - a.reach - (kRows - 1) - q.at, (int64_t)-1);
    fetch(begin);
    bool odd = put(begin, 0);
    odds |= odd;
    if (a.bias) {
      bias_behind = table[bt.size - 1];
      bias_ahead = table[0];
      if (far_off(bias_behind)) plain_from = 0x7fffffff;
      if (far_off(bias_ahead)) plain_to = -1;
    }
    for (int i0 = begin, buf = 0; i0 < end; i0 += kRows, buf ^= 1) {
      const bool next = i0 + kRows < end;
      if (next) fetch(i0 + kRows);
      if (i0 >= from_i) {
        const float mylse = stats[buf][0][lane % kRows];
        bool exact = !started, dead = false;
        if (__any(far_off(mylse))) {       // a statistic far off, or a row without one
          // Rows that are no queries are zeros, which times a key or value that is not finite are NaN: they are left out one by one.
          dead = __any(mylse == __builtin_inff()) && __any(odd_rows<Tl, KS>(fk, fv));
          exact = exact || dead || __any(mylse < __builtin_inff() && far_off(mylse));
        }
        if (!SEEN && !exact && (i0 >= plain_from || i0 <= plain_to)) tile(std::true_type(), i0, buf, false, false, false);
        else tile(std::false_type(), i0, buf, exact, odd, dead);
      }
      if (next) odd = put(i0 + kRows, buf ^ 1), odds |= odd;
    }
  }
  if (!SEEN && threadIdx.x == 0 && a.causal) a.odd[blockIdx.x] = odds;
  if (!SEEN && odds) return;
  if (j >= q.len) return;
  if (!there) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) dk[dt] = dv[dt] = (typename Tl::Acc)(0.f);
  }
  if (parts > 1) {
    float* to = a.joint + (((int64_t)part * pairs + pair) * a.Tk + j) * 2 * a.d;
    store_sums<Tl, DT>(to, dk, a.scale, a.d, lane);
    store_sums<Tl, DT>(to + a.d, dv, 1.f, a.d, lane);
    return;
  }
  if (a.dk.p) store_column<Tl, DT>(static_cast<E*>(const_cast<void*>(a.dk.p)) + (int64_t)j * a.dk.st + n * a.dk.sn + y * a.d, dk, a.scale, a.d, lane);
  if (a.dv.p) store_column<Tl, DT>(static_cast<E*>(const_cast<void*>(a.dv.p)) + (int64_t)j * a.dv.st + n * a.dv.sn + y * a.d, dv, 1.f, a.d, lane);
}

// The sum of the parts: four numbers a thread, dk and dv of a key side by side.
template <class E>
__global__ __launch_bounds__(256) void k_attn_dkv_join(Args a) {
  const int kvs = a.heads / a.group, parts = a.head_parts * a.row_parts, per = a.d / 2;      // 2 d / 4
  const int64_t keys = a.N * kvs * a.Tk, all = keys * per;
  for (int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x; x < all; x += (int64_t)gridDim.x * 256) {
    const int64_t key = x / per;
    int c = (int)(x % per) * 4;
    const int j = (int)(key % a.Tk), y = (int)(key / a.Tk % kvs);
    const int64_t n = key / a.Tk / kvs;
    const int len = a.lengths ? min(max(a.lengths[n], 0), a.Tk) : a.Tk;
    if (j >= len) continue;
    float4 s = *reinterpret_cast<const float4*>(a.joint + key * 2 * a.d + c);
    for (int k = 1; k < parts; ++k) {
      const float4 u = *reinterpret_cast<const float4*>(a.joint + (k * keys + key) * 2 * a.d + c);
      s.x += u.x; s.y += u.y; s.z += u.z; s.w += u.w;
    }
    const Rows& to = c < a.d ? a.dk : a.dv;
    if (c >= a.d) c -= a.d;
    if (!to.p) continue;
    E* at = static_cast<E*>(const_cast<void*>(to.p)) + (int64_t)j * to.st + n * to.sn + y * a.d + c;
    if constexpr (sizeof(E) == 2) *reinterpret_cast<uint2*>(at) = make_uint2(pack2(s.x, s.y), pack2(s.z, s.w));
    else *reinterpret_cast<float4*>(at) = s;
  }
}

// ---------------------------------------------------------------------------------------------------- the bias' gradient
//
// part[h][slot][x] holds sums of distance from + x: one workgroup a head and bucket sums those of the bucket, in one order, in double: 16 distances at a
// time, 16 slots.
__global__ __launch_bounds__(256) void k_attn_bias(Args a, int size, int64_t from, float* dbias) {
  __shared__ double partial[256];
  __shared__ uint8_t map[2 * kMaxReach + 1];
  const int b = blockIdx.x % a.buckets, h = blockIdx.x / a.buckets;
  for (int x = threadIdx.x; x <= 2 * a.reach; x += 256) map[x] = a.map[x];
  __syncthreads();
  double s = 0.;
  for (int x = threadIdx.x & 15; x < size; x += 16) {
    const int c = (int)min(max(from + x, -(int64_t)a.reach), (int64_t)a.reach) + a.reach;
    if (min((int)map[c], a.buckets - 1) != b) continue;
#pragma unroll 4
    for (int slot = threadIdx.x >> 4; slot < a.slots; slot += 16) s += (double)a.part[((int64_t)h * a.slots + slot) * size + x];
  }
  partial[threadIdx.x] = s;
  __syncthreads();
  for (int m = 128; m; m /= 2) {
    if ((int)threadIdx.x < m) partial[threadIdx.x] += partial[threadIdx.x + m];
    __syncthreads();
  }
  if (threadIdx.x == 0) dbias[h * a.buckets + b] = (float)partial[0];
}

// ---------------------------------------------------------------------------------------------------- launch
template <class Tl, int NT>
bool windows_back(Args& a, hipStream_t st) {
  const int e = sizeof(typename Tl::E), W = 16 * NT;
  const Rows* const all[8] = {&a.q, &a.k, &a.v, &a.o, &a.go, &a.dq, &a.dk, &a.dv};
  for (const Rows* x : all) {
    if (x->p && std::max(x->st, x->sn) >= ((int64_t)1 << 31) / e / (W + 4)) return false;      // beyond 32-bit offsets
  }
  const WindowPlan p = plan_windows(a.N, a.heads, a.d, e);
  WindowBack w{a, p.together, p.seqs, p.groups, p.together * a.d + 16 / e, p.tables};
  const int rows = p.seqs * W, cpr = p.together * a.d * e / 16, pieces = (rows * cpr + 255) / 256;
  const int need = 4 * rows * w.pitch * e + (4 * 2 * 16 * (16 + 16 / e) + 64) * e + 4 * (p.together * 2 * W + rows * p.together + rows * cpr + rows + p.seqs);
  const unsigned lds = (unsigned)std::max(need, 4 * 4 * W * 2 * W), wgs = (unsigned)(p.slots * p.groups);
  if (lds > 65536 || pieces > 2 * NT || (pieces > NT && p.together == 8)) return false;
  w.a.slots = p.slots;
#define DGC_WINDOWS(KS)                                                                                                  \
  if (p.together == 8) hipLaunchKernelGGL((k_attn_windows_back<Tl, NT, KS, NT, 2>), wgs, 256, lds, st, w);              \
  else if (pieces > NT) hipLaunchKernelGGL((k_attn_windows_back<Tl, NT, KS, 2 * NT, 1>), wgs, 256, lds, st, w);         \
  else hipLaunchKernelGGL((k_attn_windows_back<Tl, NT, KS, NT, 1>), wgs, 256, lds, st, w)
  if (a.d <= 16) {
    DGC_WINDOWS(1);
  } else if (a.d <= 32) {
    DGC_WINDOWS(2);
  } else {
    DGC_WINDOWS(4);
  }
#undef DGC_WINDOWS
  a.slots = p.slots * p.tables;
  return true;
}

template <class Tl, int NT>
void window_back(Args& a, hipStream_t st) {
  if (a.group == 1 && windows_back<Tl, NT>(a, st)) return;
  const int kvs = a.heads / a.group;
  a.slots = back_slots(true, a.N, a.heads, kvs, 0, 0);
  const unsigned grid = (unsigned)(((int64_t)a.slots * kvs + 3) / 4), lds = a.bias ? 4 * 4 * a.group * 10 * 16 * NT : 0;
  if (a.d <= 16) hipLaunchKernelGGL((k_attn_window_back<Tl, NT, 1>), grid, 256, lds, st, a);
  else if (a.d <= 32) hipLaunchKernelGGL((k_attn_window_back<Tl, NT, 2>), grid, 256, lds, st, a);
  else hipLaunchKernelGGL((k_attn_window_back<Tl, NT, 4>), grid, 256, lds, st, a);
}

template <class Tl, int KS>
void long_back(Args& a, hipStream_t st) {
  typedef typename Tl::E E;
  constexpr int M = Tl::M, LPR = (KS == 3 ? 4 : KS == 6 ? 8 : KS) * 16 / ops::Elem<E>::kPer;      // a power of two
  const int64_t rows = (int64_t)a.Tq * a.N * a.heads;
  if (rows > 0) hipLaunchKernelGGL((k_attn_delta<E, LPR>), (unsigned)std::min<int64_t>((rows * LPR + 255) / 256, 256 * 32), 256, 0, st, a);
  const unsigned lds = bias_bytes(a);
  if (rows > 0 && (a.dq.p || a.part)) {
    const int64_t blocks = (a.Tq + 4 * M - 1) / (4 * M);
    a.slots = a.part ? back_slots(false, a.N, a.heads, 0, blocks, at_once(Tl::kExact, a.d)) : (int)(a.N * blocks);
    const unsigned more = a.part ? 4 * 4 * (table_size(a.reach, a.causal) + 2 * M * M) : 0;
    hipLaunchKernelGGL((k_attn_dq<Tl, KS, false>), (unsigned)(a.slots * a.heads), 256, lds + more, st, a);
    if (a.causal && a.dq.p) hipLaunchKernelGGL((k_attn_dq<Tl, KS, true>), (unsigned)(a.slots * a.heads), 256, lds, st, a);
  }
  if (a.dk.p || a.dv.p) {
    const int64_t blocks = (a.Tk + 4 * M - 1) / (4 * M);
    const Parts p = key_parts(a.Tq, a.Tk, a.N, a.heads, a.heads / a.group, sizeof(E) == 4);
    a.head_parts = p.heads;
    a.row_parts = p.rows;
    const unsigned grid = (unsigned)(a.N * (a.heads / a.group) * blocks * p.heads * p.rows);
    hipLaunchKernelGGL((k_attn_dkv<Tl, KS, false>), grid, 256, lds, st, a);
    if (a.causal) hipLaunchKernelGGL((k_attn_dkv<Tl, KS, true>), grid, 256, lds, st, a);
    if (p.heads * p.rows > 1) {
      const int64_t threads = a.N * (a.heads / a.group) * a.Tk * (a.d / 2);
      hipLaunchKernelGGL(k_attn_dkv_join<E>, (unsigned)std::min<int64_t>((threads + 255) / 256, 256 * 32), 256, 0, st, a);
    }
  }
}

// fp32 heads are padded to 16, 32, 48, 64, 96 or 128 columns (200 x 101 tokens, 4 heads of 40: 168 us with 48 columns, 186 with 64; 40 x 512, 4 of 96: 360 and
// 440), bf16 ones, whose tiles are 32 wide, to 16, 32, 64 or 128.
template <class Tl16, class TlLong>
void backward(Args a, float* dbias, hipStream_t st) {
  int size = table_size(a.reach, a.causal);
  int64_t from = table_from(a.reach, a.causal);
  if (a.N == 0 || a.Tk == 0) {
    // no gradients but the bias' zeros
  } else if (takes_window_back(a.Tk, a.d, a.group, a.first != nullptr)) {
    const int W = a.Tk <= 16 ? 16 : 32;
    size = 2 * W;
    from = (int64_t)a.Tk - a.Tq - W + 1;
    if (W == 16) window_back<Tl16, 1>(a, st);
    else window_back<Tl16, 2>(a, st);
  } else if (a.d <= 16) {
    long_back<TlLong, 1>(a, st);
  } else if (a.d <= 32) {
    long_back<TlLong, 2>(a, st);
  } else if (a.d <= 48 && TlLong::kExact) {
    long_back<TlLong, TlLong::kExact ? 3 : 4>(a, st);
  } else if (a.d <= 64) {
    long_back<TlLong, 4>(a, st);
  } else if (a.d <= 96 && TlLong::kExact) {
    long_back<TlLong, TlLong::kExact ? 6 : 8>(a, st);
  } else {
    long_back<TlLong, 8>(a, st);
  }
  if (!a.part) a.slots = 0;
  if (dbias) hipLaunchKernelGGL(k_attn_bias, (unsigned)(a.heads * a.buckets), 256, 0, st, a, size, from, dbias);
}

}  // namespace

void attn_backward_f32(const Args& a, float* dbias, hipStream_t st) { backward<Full, Full>(a, dbias, st); }
void attn_backward_bf16(const Args& a, float* dbias, hipStream_t st) { backward<Small, Wide>(a, dbias, st); }

}  // namespace attn
}  // namespace dgc
