// Softmax attention over the tokens of sequences, backward.  With the forward pass' o and lse, for every query i and key j that it sees:
//
//   P = e^(s - lse),  dP = do_i . v_j,  D = do_i . o_i,  dS = P (dP - D)
//   dv_j = sum_i P do_i,  dq_i = scale sum_j dS k_j,  dk_j = scale sum_i dS q_i,  dbias[h][b] = sum of dS over the pairs whose distance has bucket b
//
// Scores are computed again, not kept.  In k_attn_dq queries are columns and keys are summed over, in k_attn_dkv keys are columns and queries are summed over
// (heads that share a key head one after the other), so no two workgroups add to one number: no atomics on memory, one order of sums, at the price of
// seven products for five.  k_attn_window_back has a whole window in a wave and needs five.
// Rounding: bf16 tensors enter products as they are, scores, P, dP, D and dS are fp32; P and dS are rounded to bf16 (2^-9 of themselves)
// for the products of dv, dq and dk, which are summed in fp32; the bias' gradient sums dS as it is, in fp32 and at the end in double.
//
// The bias' gradient: every wave adds dS by distance into tables of its own in LDS.  Lanes of one row of lanes hold one key (or query) and neighbouring
// queries (keys), so their distances differ; each row of lanes has a table, so an instruction never adds twice to one place, and a
// wave's instructions are taken in order: the sums have one order.  k_attn_bias joins the tables.
#include <algorithm>

#include "dgc_attn_dev.h"

namespace dgc {
namespace attn {
namespace {

__device__ __forceinline__ void add_lds(float* to, float x) { __hip_atomic_fetch_add(to, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WAVEFRONT); }

// ---------------------------------------------------------------------------------------------------- windows
template <class Tl, int NT, int KS>
__global__ __launch_bounds__(256) void k_attn_window_back(Args a) {
  typedef typename Tl::E E;
  typedef typename Tl::Frag Frag;
  constexpr int DT = Geometry<Tl, KS>::DT, P = Geometry<Tl, KS>::P, W = 16 * NT, PT = 16 + 16 / (int)sizeof(E);
  __shared__ __attribute__((aligned(16))) E room[4][(W + 32) * P + 2 * 16 * PT];
  extern __shared__ float tables[];       // with a bias: [4 waves][group][1 + 4][2 W], the bias by distance and four tables of sums
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, sub = lane >> 4, kvs = a.heads / a.group;
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
          gather<Tl, DT>(dq, sk + 16 * t * P, P, Packed<Tl>(ds), lane, odd_k, [](int) { return 0; }, [&](int c) { return c - apart; });
          gather<Tl, DT>(dv[t], sg, P, Packed<Tl>(Tl::across(sp, PT, 0, 0, lane)), lane, odd_qg, [&](int c) { return apart + c; }, [](int) { return 15; });
          gather<Tl, DT>(dk[t], sq, P, Packed<Tl>(Tl::across(ss, PT, 0, 0, lane)), lane, odd_qg, [&](int c) { return apart + c; }, [](int) { return 15; });
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
// As the forward pass: 4 M queries a workgroup, keys in tiles of 64 through LDS.
template <class Tl, int KS>
__global__ __launch_bounds__(256) void k_attn_dq(Args a) {
  typedef typename Tl::E E;
  constexpr int M = Tl::M, NT = kTile / M, DT = Geometry<Tl, KS>::DT, P = Geometry<Tl, KS>::P;
  constexpr int SETS = M == 32 ? 2 : 1;     // tables of a wave: 16-column tiles add one row of lanes after the other to one
  __shared__ __attribute__((aligned(16))) E sk[kTile * P], sv[kTile * P];
  __shared__ float seen[kTile];
  extern __shared__ float table[];          // the bias by distance, then the waves' tables of sums
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = Tl::col(lane), sub = Tl::sub(lane);
  const int blocks = (a.Tq + 4 * M - 1) / (4 * M), h = blockIdx.x % a.heads, slot = blockIdx.x / a.heads, y = h / a.group;
  const int from = a.causal ? 0 : -a.reach, tfrom = table_from(a.reach, a.causal), tsize = table_size(a.reach, a.causal);
  float* const sums = table + a.reach - from + 1;
  if (a.bias) {
    for (int x = threadIdx.x; x <= a.reach - from; x += 256) table[x] = bias_at(a, h, from + x);
    if (a.part) {
      for (int x = threadIdx.x; x < 4 * SETS * tsize; x += 256) sums[x] = 0.f;
    }
  }
  float* const mysums = sums + (wave * SETS + (SETS == 2 ? sub : 0)) * tsize;
  float behind = 0.f, ahead = 0.f;          // sums of tiles that are far off as a whole
  for (int64_t item = slot; item < a.N * blocks; item += a.slots) {
    const int64_t n = item % a.N;
    const int i0 = (int)(blocks - 1 - item / a.N) * 4 * M;
    const Seq q(a, n);
    if (i0 >= q.hi || i0 + 4 * M <= q.lo) continue;
    const int least = max(i0, q.lo), most = min(i0 + 4 * M, q.hi) - 1;
    const int kend = a.causal ? (int)min((int64_t)q.len, q.at + most + 1) : q.len;
    const int mine = i0 + wave * M, i = mine + col;
    const bool row = i >= q.lo && i < q.hi;
    const int64_t stat = (n * a.heads + h) * a.Tq + i;
    const float lse = row ? a.lse[stat] : -__builtin_inff(), D = row ? a.delta[stat] : 0.f, lse2 = lse * kLog2e;
    const bool live = lse != -__builtin_inff();
    const bool exact = Tl::kExact || __any(live && far_off(lse));
    const bool some = max(mine, q.lo) < min(mine + M, q.hi);
    const int p0 = some ? (int)(q.at + max(mine, q.lo)) : -1, p1 = some ? (int)(q.at + min(mine + M, q.hi) - 1) : -1, p = live ? (int)(q.at + i) : -1;
    typename Tl::Frag fq[KS], fg[KS];
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
    Stage<E, kTile, KS> nk, nv;
    nk.fetch(kbase, a.k.st, 0, a.d, there);
    nv.fetch(vbase, a.v.st, 0, a.d, there);
    typename Tl::Acc dq[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) dq[dt] = (typename Tl::Acc)(0.f);

    for (int j0 = 0; j0 < kend; j0 += kTile) {
      __syncthreads();
      nk.put(sk, P);
      nv.put(sv, P);
      const bool edge = a.causal && j0 + kTile - 1 > q.at + least;
      const bool masked = a.keep || j0 + kTile > kend;
      if (masked && threadIdx.x < kTile) seen[threadIdx.x] = there(j0 + (int)threadIdx.x) ? 1.f : 0.f;
      const bool slow = edge ? __syncthreads_or(nk.template odd<Tl>()) : (__syncthreads(), false);
      if (j0 + kTile < kend) {
        nk.fetch(kbase, a.k.st, j0 + kTile, a.d, there);
        nv.fetch(vbase, a.v.st, j0 + kTile, a.d, there);
      }
      if (!some || (a.causal && j0 > p1)) continue;
      const bool far = a.bias && p0 - (j0 + kTile - 1) >= a.reach, before = a.bias && p1 - j0 <= -a.reach;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int first = j0 + t * M;
        if (a.causal && first > p1) break;
        typename Tl::Acc x = (typename Tl::Acc)(0.f), z = x;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          x = Tl::mma(Tl::rows(sk + t * M * P, P, s, lane), fq[s], x);
          z = Tl::mma(Tl::rows(sv + t * M * P, P, s, lane), fg[s], z);
        }
        if (!a.bias || far || before) {
          const float b = !a.bias ? 0.f : table[far ? a.reach - from : 0];
#pragma unroll
          for (int r = 0; r < Tl::NR; ++r) x[r] = fmaf(x[r], a.scale, b);
        } else {
#pragma unroll
          for (int r = 0; r < Tl::NR; ++r) x[r] = fmaf(x[r], a.scale, table[min(max(p - (first + Tl::row(r, lane)), from), a.reach) - from]);
        }
        const bool holes = masked || (a.causal && first + M - 1 > p0) || !__all(live);
        if (holes) {
#pragma unroll
          for (int r = 0; r < Tl::NR; ++r) {
            const int j = first + Tl::row(r, lane);
            const bool out = !live || (a.causal && j > p) || (masked && seen[j - j0] == 0.f);
            x[r] = out ? 0.f : weight(x[r], lse, lse2, exact);
            z[r] = out ? 0.f : x[r] * (z[r] - D);
          }
        } else {
#pragma unroll
          for (int r = 0; r < Tl::NR; ++r) z[r] = weight(x[r], lse, lse2, exact) * (z[r] - D);
        }
        if (a.part) {
          if (far || before) {
            float s = 0.f;
#pragma unroll
            for (int r = 0; r < Tl::NR; ++r) s += z[r];
            (far ? behind : ahead) += s;
          } else {
#pragma unroll
            for (int r = 0; r < Tl::NR; ++r) {
              const int away = p - (first + Tl::row(r, lane)) - tfrom;
              if constexpr (SETS == 2) {
                if (z[r] != 0.f) add_lds(mysums + away, z[r]);
              } else {
                for (int s = 0; s < Tl::SUBS; ++s) {
                  if (s == sub && z[r] != 0.f) add_lds(mysums + away, z[r]);
                }
              }
            }
          }
        }
        gather<Tl, DT>(dq, sk + t * M * P, P, Packed<Tl>(z), lane, slow, [](int) { return 0; }, [&](int c) { return (int)(q.at + mine + c) - first; });
      }
    }
    if (row && a.dq.p) {
      if (!live) {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) dq[dt] = (typename Tl::Acc)(0.f);
      }
      store_column<Tl, DT>(static_cast<E*>(const_cast<void*>(a.dq.p)) + (int64_t)i * a.dq.st + n * a.dq.sn + h * a.d, dq, a.scale, a.d, lane);
    }
    __syncthreads();      // before the next item's keys
  }
  if (a.part) {
    __syncthreads();
    behind = wave_sum(behind);
    ahead = wave_sum(ahead);
    if (lane == 0) {
      sums[wave * SETS * tsize + a.reach - tfrom] += behind;
      if (!a.causal) sums[wave * SETS * tsize - a.reach - tfrom] += ahead;
    }
    __syncthreads();
    for (int x = threadIdx.x; x < tsize; x += 256) {
      float s = 0.f;
      for (int w = 0; w < 4 * SETS; ++w) s += sums[w * tsize + x];
      a.part[((int64_t)h * a.slots + slot) * tsize + x] = s;
    }
  }
}

// ---------------------------------------------------------------------------------------------------- dk, dv
//
// A workgroup takes 4 M keys of one sequence and key head, a wave M of them in registers, and walks over the queries that see them in tiles of
// 64 that lie in LDS, for one head that shares the keys after the other.
template <class Tl, int KS>
__global__ __launch_bounds__(256) void k_attn_dkv(Args a) {
  typedef typename Tl::E E;
  constexpr int M = Tl::M, NT = kTile / M, DT = Geometry<Tl, KS>::DT, P = Geometry<Tl, KS>::P;
  __shared__ __attribute__((aligned(16))) E sq[kTile * P], sg[kTile * P];
  __shared__ __attribute__((aligned(16))) float slse[kTile], sD[kTile];
  extern __shared__ float table[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = Tl::col(lane), sub = Tl::sub(lane), kvs = a.heads / a.group;
  const uint32_t pairs = (uint32_t)(a.N * kvs), pair = blockIdx.x % pairs;
  const int64_t n = pair / kvs;
  const int y = pair % kvs, k0 = (int)(blockIdx.x / pairs) * 4 * M;
  const Seq q(a, n);
  if (k0 >= q.len) return;
  const int mine = k0 + wave * M, j = mine + col;
  const bool there = j < q.len && (!a.keep || a.keep[(int64_t)j * a.N + n]);
  const int from = a.causal ? 0 : -a.reach;
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
  const int begin = a.causal ? (int)min((int64_t)q.hi, max((int64_t)q.lo, k0 - q.at)) : q.lo;      // the first query that sees one of these keys
  for (int g = 0; g < a.group; ++g) {
    const int h = y * a.group + g;
    __syncthreads();
    if (a.bias) {
      for (int x = threadIdx.x; x <= a.reach - from; x += 256) table[x] = bias_at(a, h, from + x);
    }
    const E* qbase = static_cast<const E*>(a.q.p) + n * a.q.sn + h * a.d;
    const E* gbase = static_cast<const E*>(a.go.p) + n * a.go.sn + h * a.d;
    const float* lses = a.lse + (n * a.heads + h) * a.Tq;
    const float* Ds = a.delta + (n * a.heads + h) * a.Tq;
    // A query that sees nothing gives no gradient: its rows are zero, whatever they hold.
    auto live = [&](int i) { return i >= q.lo && i < q.hi && lses[i] != -__builtin_inff(); };
    Stage<E, kTile, KS> nq, ng;
    float nlse = 0.f, nD = 0.f;
    auto fetch = [&](int i0) {
      nq.fetch(qbase, a.q.st, i0, a.d, live);
      ng.fetch(gbase, a.go.st, i0, a.d, live);
      if (threadIdx.x < kTile) {
        const int i = i0 + threadIdx.x;
        const bool ok = live(i);
        nlse = ok ? lses[i] : __builtin_inff();      // its weights are zero
        nD = ok ? Ds[i] : 0.f;
      }
    };
    if (begin < q.hi) fetch(begin);
    for (int i0 = begin; i0 < q.hi; i0 += kTile) {
      __syncthreads();
      nq.put(sq, P);
      ng.put(sg, P);
      if (threadIdx.x < kTile) slse[threadIdx.x] = nlse, sD[threadIdx.x] = nD;
      const bool edge = a.causal && q.at + i0 < k0 + 4 * M - 1;
      const bool slow = edge ? __syncthreads_or(nq.template odd<Tl>() || ng.template odd<Tl>()) : (__syncthreads(), false);
      if (i0 + kTile < q.hi) fetch(i0 + kTile);
      const int first_p = (int)(q.at + i0);
      if (mine >= q.len || (a.causal && first_p + kTile - 1 < mine)) continue;
      const float mylse = slse[lane];
      const bool exact = Tl::kExact || __any(mylse < __builtin_inff() && far_off(mylse));
      const bool far = a.bias && first_p - (mine + M - 1) >= a.reach, before = a.bias && first_p + kTile - 1 - mine <= -a.reach;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int pt = first_p + t * M;
        if (a.causal && pt + M - 1 < mine) continue;
        typename Tl::Acc x = (typename Tl::Acc)(0.f), z = x;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          x = Tl::mma(Tl::rows(sq + t * M * P, P, s, lane), fk[s], x);
          z = Tl::mma(Tl::rows(sg + t * M * P, P, s, lane), fv[s], z);
        }
        if (!a.bias || far || before) {
          const float b = !a.bias ? 0.f : table[far ? a.reach - from : 0];
#pragma unroll
          for (int r = 0; r < Tl::NR; ++r) x[r] = fmaf(x[r], a.scale, b);
        } else {
#pragma unroll
          for (int r = 0; r < Tl::NR; ++r) x[r] = fmaf(x[r], a.scale, table[min(max(pt + Tl::row(r, lane) - j, from), a.reach) - from]);
        }
        const bool holes = a.causal && pt < mine + M - 1;
#pragma unroll
        for (int r = 0; r < Tl::NR; r += 4) {
          const float4 l4 = *reinterpret_cast<const float4*>(slse + t * M + Tl::row(r, lane));
          const float4 d4 = *reinterpret_cast<const float4*>(sD + t * M + Tl::row(r, lane));
          const float ls[4] = {l4.x, l4.y, l4.z, l4.w}, ds[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[r + e] = weight(x[r + e], ls[e], ls[e] * kLog2e, exact);
            z[r + e] = x[r + e] * (z[r + e] - ds[e]);
          }
        }
        if (holes) {
#pragma unroll
          for (int r = 0; r < Tl::NR; ++r) {
            const bool out = pt + Tl::row(r, lane) < j;
            x[r] = out ? 0.f : x[r];
            z[r] = out ? 0.f : z[r];
          }
        }
        auto lo = [&](int c) { return mine + c - pt; };
        auto hi = [](int) { return M - 1; };
        gather<Tl, DT>(dv, sg + t * M * P, P, Packed<Tl>(x), lane, slow, lo, hi);
        gather<Tl, DT>(dk, sq + t * M * P, P, Packed<Tl>(z), lane, slow, lo, hi);
      }
    }
  }
  if (j >= q.len) return;
  if (!there) {
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) dk[dt] = dv[dt] = (typename Tl::Acc)(0.f);
  }
  if (a.dk.p) store_column<Tl, DT>(static_cast<E*>(const_cast<void*>(a.dk.p)) + (int64_t)j * a.dk.st + n * a.dk.sn + y * a.d, dk, a.scale, a.d, lane);
  if (a.dv.p) store_column<Tl, DT>(static_cast<E*>(const_cast<void*>(a.dv.p)) + (int64_t)j * a.dv.st + n * a.dv.sn + y * a.d, dv, 1.f, a.d, lane);
}

// ---------------------------------------------------------------------------------------------------- the bias' gradient
//
// part[h][slot][x] holds sums of distance from + x: one workgroup a head and bucket sums those of the bucket, in one order, in double.
__global__ __launch_bounds__(256) void k_attn_bias(Args a, int size, int64_t from, float* dbias) {
  __shared__ double partial[256];
  const int b = blockIdx.x % a.buckets, h = blockIdx.x / a.buckets;
  double s = 0.;
  for (int x = 0; x < size; ++x) {
    const int c = (int)min(max(from + x, -(int64_t)a.reach), (int64_t)a.reach) + a.reach;
    if (min((int)a.map[c], a.buckets - 1) != b) continue;
    for (int slot = threadIdx.x; slot < a.slots; slot += 256) s += (double)a.part[((int64_t)h * a.slots + slot) * size + x];
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
void window_back(Args& a, hipStream_t st) {
  const int kvs = a.heads / a.group;
  a.slots = back_slots(true, a.N, a.heads, kvs, 0);
  const unsigned grid = (unsigned)(((int64_t)a.slots * kvs + 3) / 4), lds = a.bias ? 4 * 4 * a.group * 10 * 16 * NT : 0;
  if (a.d <= 16) hipLaunchKernelGGL((k_attn_window_back<Tl, NT, 1>), grid, 256, lds, st, a);
  else if (a.d <= 32) hipLaunchKernelGGL((k_attn_window_back<Tl, NT, 2>), grid, 256, lds, st, a);
  else hipLaunchKernelGGL((k_attn_window_back<Tl, NT, 4>), grid, 256, lds, st, a);
}

template <class Tl, int KS>
void long_back(Args& a, hipStream_t st) {
  typedef typename Tl::E E;
  constexpr int M = Tl::M, LPR = KS * 16 / ops::Elem<E>::kPer;
  const int64_t rows = (int64_t)a.Tq * a.N * a.heads;
  if (rows > 0) hipLaunchKernelGGL((k_attn_delta<E, LPR>), (unsigned)std::min<int64_t>((rows * LPR + 255) / 256, 256 * 32), 256, 0, st, a);
  const unsigned lds = a.bias ? 4 * (a.causal ? a.reach + 1 : 2 * a.reach + 1) : 0;
  if (rows > 0 && (a.dq.p || a.part)) {
    const int64_t blocks = (a.Tq + 4 * M - 1) / (4 * M);
    a.slots = a.part ? back_slots(false, a.N, a.heads, 0, blocks) : (int)(a.N * blocks);
    const unsigned more = a.part ? 4 * 4 * (M == 32 ? 2 : 1) * table_size(a.reach, a.causal) : 0;
    hipLaunchKernelGGL((k_attn_dq<Tl, KS>), (unsigned)(a.slots * a.heads), 256, lds + more, st, a);
  }
  if (a.dk.p || a.dv.p) {
    const int64_t blocks = (a.Tk + 4 * M - 1) / (4 * M);
    hipLaunchKernelGGL((k_attn_dkv<Tl, KS>), (unsigned)(a.N * (a.heads / a.group) * blocks), 256, lds, st, a);
  }
}

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
  } else if (a.d <= 64) {
    long_back<TlLong, 4>(a, st);
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
