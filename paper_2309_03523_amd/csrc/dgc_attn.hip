// Softmax attention over the tokens of sequences, forward.  For query i of sequence n, at position p = at + i, and head h:
//
//   s_j = scale q_i . k_j + bias[h][map[p - j]]  over the keys that it sees,  lse = log sum e^s_j,  o = sum e^(s_j - lse) v_j
//
// Scores are formed turned, keys in rows and queries in columns: a lane then holds scores of one query, the running maximum and sum of
// its softmax are two registers, and the probabilities are the right operand of the product with the values as they stand.
// Rounding: bf16 tensors enter products as they are; scores, exponents, maxima and sums are fp32; probabilities are rounded
// to bf16 (by up to 2^-8 of themselves) for their product with the values, which is summed in fp32 (k_attn_few, on the vector
// unit, keeps them in fp32).  fp32 tensors: fp32 throughout.
//
// Kernels, by the lengths alone.  Up to 64 keys, a wave a sequence and head: k_attn_windows (up to 32 keys, queries of all sequences at one
// position, rows that fit 64 KB of LDS) and k_attn_window (the rest).  Else up to 16 queries, keys split among lanes, waves and workgroups and joined by k_attn_join:
// k_attn_few (one or two rows that share a key head) and k_attn_rows (more, on the matrix unit).  k_attn_forward: the rest.
#include <algorithm>
#include <type_traits>

#include "dgc_attn_dev.h"

namespace dgc {
namespace attn {
namespace {

// ---------------------------------------------------------------------------------------------------- long sequences
//
// A workgroup takes 4 M queries of one sequence and head, a wave M of them, and walks over the keys in tiles of 64 (fp32, wide bf16 heads: 32) that lie in LDS
// once for all four; the next tile's rows are on their way in registers meanwhile.  What bounds it are the vector instructions of the softmax: four sequences of 8192
// tokens, 8 heads of 64, bf16 take 0.40 ms (0.47 in a card's first passes) where the products alone would take 0.23; vector units are busy for 63 % of that, the matrix units for 29 %.
// Tiles without masks, of one bias, therefore have a path without branches and with one multiply-add a score (with a mask, where none is, 0.78 ms).
template <class Tl, int KS>
__global__ __launch_bounds__(256, 2) void k_attn_forward(Args a) {
  typedef typename Tl::E E;
  constexpr int M = Tl::M, NT = Geometry<Tl, KS>::NT, kKeys = NT * M, DT = Geometry<Tl, KS>::DT, P = Geometry<Tl, KS>::P;
  __shared__ __attribute__((aligned(16))) E room[2][2 * kKeys * P];
  __shared__ float seens[2][kKeys];      // 0 where a key is masked
  extern __shared__ float table[];       // bias by distance
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = Tl::col(lane), sub = Tl::sub(lane);
  const uint32_t pairs = (uint32_t)(a.N * a.heads), blocks = (uint32_t)((a.Tq + 4 * M - 1) / (4 * M));
  // The workgroups of a sequence and head lie `pairs` apart: on one chiplet's L2 where pairs are a multiple of 8.  The longest walks first.
  const uint32_t pair = blockIdx.x % pairs;
  const int64_t n = pair / a.heads;
  const int h = pair % a.heads, y = h / a.group;
  const int i0 = (int)(blocks - 1 - blockIdx.x / pairs) * 4 * M;
  const Seq q(a, n);
  if (i0 >= q.hi || i0 + 4 * M <= q.lo) return;
  const int least = max(i0, q.lo), most = min(i0 + 4 * M, q.hi) - 1;      // live queries of the workgroup
  const int kend = a.causal ? (int)min((int64_t)q.len, q.at + most + 1) : q.len;
  const int mine = i0 + wave * M, i = mine + col;
  const bool live = i >= q.lo && i < q.hi;
  // The positions of this wave's first and last live query, and the lane's own; where none is live, as of a query that sees nothing.
  const bool some = max(mine, q.lo) < min(mine + M, q.hi);
  const int p0 = some ? (int)(q.at + max(mine, q.lo)) : -1, p1 = some ? (int)(q.at + min(mine + M, q.hi) - 1) : -1, p = live ? (int)(q.at + i) : -1;

  const BiasTable bt(a);
  if (a.bias) bt.fill(a, table, h, true);
  const float* const mytable = table + (a.reach + kPast) - (live ? p : p0) + 4 * sub;      // plus a key's place
  typename Tl::Frag fq[KS];
  {
    const E* row = static_cast<const E*>(a.q.p) + (int64_t)i * a.q.st + n * a.q.sn + h * a.d;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int c = 16 * s + Tl::KE * sub;
      fq[s] = live && c < a.d ? *reinterpret_cast<const typename Tl::Frag*>(row + c) : Tl::zero();
    }
  }
  const E* kbase = static_cast<const E*>(a.k.p) + n * a.k.sn + y * a.d;
  const E* vbase = static_cast<const E*>(a.v.p) + n * a.v.sn + y * a.d;
  auto there = [&](int j) { return j < kend && (!a.keep || a.keep[(int64_t)j * a.N + n]); };
  // Where tiles change their kind, so that one comparison tells it.  No key of a tile that ends by `whole` is masked; every query of the workgroup
  // sees those up to `inside`; `plain_to`, `plain_from`: this wave's queries see the whole tile, with one bias, ahead or behind the reach.
  const int whole = a.keep ? 0 : kend, inside = a.causal ? (int)(q.at + least) + 1 : kend + kKeys;
  int plain_to = Tl::kExact || !(a.scale > 0.f) ? 0 : min(whole, min(a.causal ? p0 + 1 : kend, a.bias ? p0 - a.reach + 1 : kend));
  int plain_from = Tl::kExact || !(a.scale > 0.f) || a.causal ? 0x7fffffff : p1 + a.reach;
  auto holes = [&](int j0) { return j0 + kKeys > whole; };
  Stage<E, kKeys, KS> nk, nv;
  nk.init(a.k.st, a.d);
  nv.init(a.v.st, a.d);
  const bool near = nk.near && nv.near;
  const E *knext = kbase, *vnext = vbase;
  const int64_t kstep = kKeys * a.k.st, vstep = kKeys * a.v.st;
  auto fetch = [&](int j0) __attribute__((always_inline)) {
    if (!holes(j0) && near) {
      nk.fetch_all(knext);
      nv.fetch_all(vnext);
      knext += kstep;
      vnext += vstep;
    } else {
      nk.fetch(kbase, a.k.st, j0, there);
      nv.fetch(vbase, a.v.st, j0, there);
    }
  };
  // Lays out a tile; whether a zero weight would meet a value of it that is not finite.
  auto put = [&](int j0, int b) __attribute__((always_inline)) -> bool {
    nk.put(room[b], P);
    nv.put(room[b] + kKeys * P, P);
    if (holes(j0) && threadIdx.x < kKeys) seens[b][threadIdx.x] = there(j0 + (int)threadIdx.x) ? 1.f : 0.f;
    if (j0 + kKeys > inside) return __syncthreads_or(nv.template odd<Tl>());
    __syncthreads();
    return false;
  };
  typename Tl::Acc o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) o[dt] = (typename Tl::Acc)(0.f);
  float m = -__builtin_inff(), l = 0.f;
  // One tile.  PLAIN: every query sees all of it, with one bias, and scale > 0: scores stay as the product left them, a score's weight is one
  // multiply-add and one power of two, and nothing branches, so products and weights of the tile's halves run side by side.
  // SEEN: values that are not finite reach only those that see them.
  float bias_behind = 0.f, bias_ahead = 0.f;       // beyond the reach
  auto tile = [&](auto plain, auto seen_only, int j0, int buf) __attribute__((always_inline)) {
    constexpr bool PLAIN = decltype(plain)::value, SEEN = decltype(seen_only)::value;
    const E *sk = room[buf], *sv = sk + kKeys * P;
    typename Tl::Acc x[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      x[t] = (typename Tl::Acc)(0.f);
#pragma unroll
      for (int s = 0; s < KS; ++s) x[t] = Tl::mma(Tl::rows(sk + t * M * P, P, s, lane), fq[s], x[t]);
    }
    const bool behind = p0 - (j0 + kKeys - 1) >= a.reach, ahead = p1 - j0 <= -a.reach;      // all of it as far as the reach
    const float one = behind ? bias_behind : bias_ahead;
    float mult = 1.f, add = 0.f;       // scores are x mult + add
    if (PLAIN) {
      mult = a.scale;
      add = one;
    } else if (!a.bias || behind || ahead) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int r = 0; r < Tl::NR; ++r) x[t][r] = fmaf(x[t][r], a.scale, one);
      }
    } else {
      const float* const at = mytable + j0;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int r = 0; r < Tl::NR; ++r) x[t][r] = fmaf(x[t][r], a.scale, at[t * M + Tl::row(r)]);
      }
    }
    if (!PLAIN && holes(j0)) {
      const float* seen = seens[buf] + 4 * sub;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int r = 0; r < Tl::NR; ++r) x[t][r] = seen[t * M + Tl::row(r)] == 0.f ? -__builtin_inff() : x[t][r];
      }
    }
    if (!PLAIN && a.causal && j0 + kKeys - 1 > p0) {
      const int upto = p - j0 - 4 * sub;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int r = 0; r < Tl::NR; ++r) x[t][r] = t * M + Tl::row(r) > upto ? -__builtin_inff() : x[t][r];
      }
    }
    float top = x[0][0];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int r = 0; r < Tl::NR; ++r) top = fmaxf(top, x[t][r]);
    }
    top = fmaxf(m, fmaf(column_max<Tl::SUBS>(top), mult, add));
    const float off = top == -__builtin_inff() ? 0.f : top;        // no key seen so far: all terms are zero
    const float f = exp2_((m - off) * kLog2e);
    m = top;
    if (PLAIN && __any(far_off(off))) {      // so large that the multiply-add below could leave exponents far above 0
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int r = 0; r < Tl::NR; ++r) x[t][r] = exp2_((fmaf(x[t][r], mult, add) - off) * kLog2e);
      }
    } else if (PLAIN) {
      mult *= kLog2e;
      add = (add - off) * kLog2e;
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int r = 0; r < Tl::NR; ++r) x[t][r] = exp2_(fmaf(x[t][r], mult, add));
      }
    } else {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int r = 0; r < Tl::NR; ++r) x[t][r] = exp2_((x[t][r] - off) * kLog2e);
      }
    }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] *= f;
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int r = 0; r < Tl::NR; ++r) sum += x[t][r];
    }
    l = fmaf(l, f, sum);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      if (SEEN) gather_seen<Tl, DT>(o, sv + t * M * P, P, Packed<Tl>(x[t]), lane, [](int) { return 0; }, [&](int c) { return (int)(q.at + mine + c) - j0 - t * M; });
      else gather<Tl, DT>(o, sv + t * M * P, P, Packed<Tl>(x[t]), lane);
    }
  };
  const int last = !some ? -1 : a.causal ? p1 : kend;
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
    if (j0 <= last && !odd) {      // this wave's queries see something of it
      if (j0 + kKeys <= plain_to || (j0 >= plain_from && j0 + kKeys <= whole)) tile(std::true_type(), std::false_type(), j0, buf);
      else tile(std::false_type(), std::false_type(), j0, buf);
    }
    if (next) odd = put(j0 + kKeys, buf ^ 1), odds |= odd;
  }
  if (odds) {      // what was left out
    for (int j0 = 0; j0 < kend; j0 += kKeys) {
      if (j0 + kKeys <= inside) continue;
      nk.fetch(kbase, a.k.st, j0, there);
      nv.fetch(vbase, a.v.st, j0, there);
      __syncthreads();
      if (put(j0, 0) && j0 <= last) tile(std::false_type(), std::true_type(), j0, 0);
    }
  }
  l = column_sum<Tl::SUBS>(l);
  if (!live) return;
  E* row = static_cast<E*>(const_cast<void*>(a.o.p)) + (int64_t)i * a.o.st + n * a.o.sn + h * a.d;
  store_column<Tl, DT>(row, o, l == 0.f ? 0.f : 1.f / l, a.d, lane);
  if (a.lse && sub == 0) a.lse[(n * a.heads + h) * a.Tq + i] = log_sum(m, l);
}

// ---------------------------------------------------------------------------------------------------- windows
//
// Up to 16 NT keys and queries: a wave takes one sequence and head after the other, of one head, so that the table of
// its bias stays.  Queries and keys go from memory into operands; only the values pass through LDS, in the wave's own part: no wave waits for another.  10 000 x 64, 4 heads of 32:
// bf16 225 us, 3.0 TB/s, fp32 333 us, 4.0 TB/s.
template <class Tl, int NT, int KS>
__global__ __launch_bounds__(256) void k_attn_window(Args a) {
  typedef typename Tl::E E;
  typedef typename Tl::Frag Frag;
  constexpr int DT = Geometry<Tl, KS>::DT, P = Geometry<Tl, KS>::P, W = 16 * NT;
  __shared__ __attribute__((aligned(16))) E values[4][W * P];
  __shared__ float tables[4][2 * W];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane & 15, sub = lane >> 4;
  const int64_t id = (int64_t)blockIdx.x * 4 + wave;
  const int h = (int)(id % a.heads), y = h / a.group;
  int64_t n = id / a.heads;
  if (n >= a.slots) return;
  E* sv = values[wave];
  float* table = tables[wave];        // of distance at - W + 1 + x
  for (bool begun = false; n < a.N; n += a.slots) {
    const Seq q(a, n);
    if (a.bias && (a.first || !begun)) {
      for (int x = lane; x < 2 * W - 1; x += 64) table[x] = bias_at(a, h, q.at - W + 1 + x);
    }
    begun = true;
    if (q.lo >= q.hi) continue;
    // A key behind every query counts as masked, whatever it holds.
    const bool there = lane < q.len && (!a.causal || lane < q.at + q.hi) && (!a.keep || a.keep[(int64_t)lane * a.N + n]);
    const uint64_t keys = __ballot(there);
    Frag fk[NT][KS];
    bool bad = false;
    const E* qbase = static_cast<const E*>(a.q.p) + n * a.q.sn + h * a.d;
    const E* kbase = static_cast<const E*>(a.k.p) + n * a.k.sn + y * a.d;
    const E* vbase = static_cast<const E*>(a.v.p) + n * a.v.sn + y * a.d;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int j = 16 * t + col;
      const bool in = keys >> j & 1;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int c = 16 * s + 4 * sub;
        const bool ok = in && c < a.d;
        fk[t][s] = ok ? Tl::load(kbase + j * a.k.st + c) : Tl::zero();
        const Frag fv = ok ? Tl::load(vbase + j * a.v.st + c) : Tl::zero();
        bad = bad || Tl::odd(fv);
        Tl::store(sv + j * P + c, fv);
      }
    }
    wave_fence();
    const bool slow = a.causal && __any(bad);
    for (int i0 = 0; i0 < q.hi; i0 += 16) {
      if (i0 + 16 <= q.lo) continue;
      const int i = i0 + col;
      const bool live = i >= q.lo && i < q.hi;
      const int p = live ? (int)(q.at + i) : -1;
      const int last = a.causal ? (int)(q.at + min(i0 + 16, q.hi) - 1) : q.len - 1;     // the last key that one of them sees
      // The keys that this lane's query sees, one bit each.
      const uint64_t mine = !live ? 0 : a.causal && p < 63 ? keys & ((2ull << p) - 1) : keys;
      Frag fq[KS];
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const int c = 16 * s + 4 * sub;
        fq[s] = live && c < a.d ? Tl::load(qbase + i * a.q.st + c) : Tl::zero();
      }
      floatx4 x[NT];
      float top = -__builtin_inff();
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        if (16 * t > last) break;
        x[t] = (floatx4)(0.f);
#pragma unroll
        for (int s = 0; s < KS; ++s) x[t] = Tl::mma(fk[t][s], fq[s], x[t]);
        const uint32_t bits = (uint32_t)(mine >> (16 * t + 4 * sub));
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int j = 16 * t + 4 * sub + r;
          float v = x[t][r] * a.scale;
          if (a.bias) v = fmaf(x[t][r], a.scale, table[i - j + W - 1]);
          x[t][r] = bits >> r & 1 ? v : -__builtin_inff();
          top = fmaxf(top, x[t][r]);
        }
      }
      top = column_max<4>(top);
      float l = 0.f;
      floatx4 o[DT];
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) o[dt] = (floatx4)(0.f);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        if (16 * t > last) break;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          x[t][r] = weight_of(x[t][r], top);
          l += x[t][r];
        }
        if (!slow) gather<Tl, DT>(o, sv + 16 * t * P, P, Packed<Tl>(x[t]), lane);
        else gather_seen<Tl, DT>(o, sv + 16 * t * P, P, Packed<Tl>(x[t]), lane, [](int) { return 0; }, [&](int c) { return (int)(q.at + i0 + c) - 16 * t; });
      }
      l = column_sum<4>(l);
      if (!live) continue;
      E* row = static_cast<E*>(const_cast<void*>(a.o.p)) + (int64_t)i * a.o.st + n * a.o.sn + h * a.d;
      store_column<Tl, DT>(row, o, l == 0.f ? 0.f : 1.f / l, a.d, lane);
      if (a.lse && sub == 0) a.lse[(n * a.heads + h) * a.Tq + i] = log_sum(top, l);
    }
    wave_fence();
  }
}

// The same for up to 32 keys where all sequences' queries stand at one position, as a batch of windows has it, and the rows below fit 64 KB of LDS: all with up to 16 keys,
// with more not bf16 heads of 40, 64, 120 and 128 (four heads and more) and fp32 ones of 32, 64 and 128, for which two sequences, or 256 bytes, are too much (20 000 x 32, 8
// heads of 64, bf16: 890 us in k_attn_window, 3.0 TB/s; 4 of 32, fp32: 301 us, 4.4 TB/s).  What bounds it is how many pieces of
// memory a load touches: operands straight from memory are 32 bytes of each of 16 rows, and ran at 2.4 TB/s.  So a workgroup takes the rows of `together`
// neighbouring heads, up to 256 bytes, of one or two sequences as they lie, through LDS, and its waves a sequence and head each from there; the outputs go back
// the same way: 100 000 windows of 16, 8 heads of 16, bf16 in 0.385 ms, 4.4 TB/s (0.41 in a card's first passes).  The next rows are on their way meanwhile; outputs leave after they have come and before more are asked for: memory answers in
// order, so rows asked for before a store would come after it.
struct WindowArgs {
  Args a;
  int32_t together, seqs, groups;      // heads, sequences of a workgroup at a time; groups of heads
  int32_t pitch;                       // of a row in LDS
};
template <class Tl, int NT, int KS, int NC>      // NC: pieces of 16 bytes of a tensor that a thread takes
__global__ __launch_bounds__(256, NT == 1 && KS < 8 ? 4 : 2) void k_attn_windows(WindowArgs w) {
  typedef typename Tl::E E;
  typedef typename Tl::Frag Frag;
  const Args& a = w.a;
  constexpr int DT = Geometry<Tl, KS>::DT, W = 16 * NT, PER = 16 / (int)sizeof(E);
  extern __shared__ __attribute__((aligned(16))) char window_room[];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane & 15, sub = lane >> 4;
  const int group = blockIdx.x % w.groups, slot = blockIdx.x / w.groups, h0 = group * w.together, heads = min(w.together, a.heads - h0), at = a.Tk - a.Tq;
  const int y0 = h0 / a.group, kvs = (h0 + heads - 1) / a.group - y0 + 1;
  const int P = w.pitch, rows = w.seqs * W;
  E *sk = reinterpret_cast<E*>(window_room), *sv = sk + rows * P, *sq = sv + rows * P, *so = sq + rows * P;
  float* add = reinterpret_cast<float*>(so + rows * P);       // [together][2 W]: the bias by distance, -inf where the position masks
  int* there = reinterpret_cast<int*>(add + w.together * 2 * W);      // [seqs][W]: whether a key is there
  int* lens = there + rows;
  for (int x = threadIdx.x; x < rows * P; x += 256) sv[x] = 0;       // rows behind Tk meet weights of zero
  __syncthreads();
  for (int x = threadIdx.x; x < heads * 2 * W; x += 256) {
    const int away = at + x % (2 * W) - W + 1;
    add[x] = a.causal && away < 0 ? -__builtin_inff() : a.bias ? bias_at(a, h0 + x / (2 * W), away) : 0.f;
  }
  // A thread's pieces of 16 bytes: where in LDS, how far from the first sequence's first row, which sequence and row.
  const int kcpr = kvs * a.d / PER, qcpr = heads * a.d / PER, kpieces = w.seqs * a.Tk * kcpr, qpieces = w.seqs * a.Tq * qcpr;
  uint32_t koff[NC], voff[NC], qoff[NC], ooff[NC];
  int kat[NC], qat[NC], kseq[NC], krow[NC], qseq[NC], qrow[NC];
#pragma unroll
  for (int i = 0; i < NC; ++i) {
    const int c = threadIdx.x + 256 * i;
    const int kr = c / kcpr, kx = (c % kcpr) * PER, qr = c / qcpr, qx = (c % qcpr) * PER;
    kseq[i] = c < kpieces ? kr / a.Tk : w.seqs;
    krow[i] = kr % a.Tk;
    kat[i] = (kseq[i] * W + krow[i]) * P + kx;
    koff[i] = (uint32_t)((kseq[i] * a.k.sn + krow[i] * a.k.st + kx) * sizeof(E));
    voff[i] = (uint32_t)((kseq[i] * a.v.sn + krow[i] * a.v.st + kx) * sizeof(E));
    qseq[i] = c < qpieces ? qr / max(a.Tq, 1) : w.seqs;
    qrow[i] = qr % max(a.Tq, 1);
    qat[i] = (qseq[i] * W + qrow[i]) * P + qx;
    qoff[i] = (uint32_t)((qseq[i] * a.q.sn + qrow[i] * a.q.st + qx) * sizeof(E));
    ooff[i] = (uint32_t)((qseq[i] * a.o.sn + qrow[i] * a.o.st + qx) * sizeof(E));
  }
  const bool whole = a.Tk == W && a.d == 16 * KS;
  uint4 nk[NC], nv[NC], nq[NC];
  uint32_t nkeep = 0;
  int nlen = 0;
  auto fetch = [&](int64_t n0) __attribute__((always_inline)) {
    const int here = (int)min((int64_t)w.seqs, a.N - n0);
    const char* kb = reinterpret_cast<const char*>(static_cast<const E*>(a.k.p) + n0 * a.k.sn + y0 * a.d);
    const char* vb = reinterpret_cast<const char*>(static_cast<const E*>(a.v.p) + n0 * a.v.sn + y0 * a.d);
    const char* qb = reinterpret_cast<const char*>(static_cast<const E*>(a.q.p) + n0 * a.q.sn + h0 * a.d);
    nkeep = 0;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      bool in = kseq[i] < here;
      if (a.lengths) in = in && krow[i] < a.lengths[n0 + min(kseq[i], here - 1)];
      if (a.keep) in = in && a.keep[krow[i] * a.N + n0 + min(kseq[i], here - 1)];
      nkeep |= in ? 1u << i : 0;
      nk[i] = in ? *reinterpret_cast<const uint4*>(kb + koff[i]) : make_uint4(0, 0, 0, 0);
      nv[i] = in ? *reinterpret_cast<const uint4*>(vb + voff[i]) : make_uint4(0, 0, 0, 0);
      nq[i] = qseq[i] < here ? *reinterpret_cast<const uint4*>(qb + qoff[i]) : make_uint4(0, 0, 0, 0);
    }
    if ((int)threadIdx.x < w.seqs) nlen = (int)threadIdx.x >= here ? 0 : a.lengths ? min(max(a.lengths[n0 + threadIdx.x], 0), a.Tk) : a.Tk;
  };
  auto leave = [&](int64_t n0) __attribute__((always_inline)) {      // the outputs, as they lie in LDS, of queries that are tokens
    char* ob = reinterpret_cast<char*>(static_cast<E*>(const_cast<void*>(a.o.p)) + n0 * a.o.sn + h0 * a.d);
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      if (qseq[i] < w.seqs && at + qrow[i] < lens[qseq[i]]) *reinterpret_cast<uint4*>(ob + ooff[i]) = *reinterpret_cast<const uint4*>(so + qat[i]);
    }
  };
  const int64_t step = (int64_t)a.slots * w.seqs;
  int64_t n0 = (int64_t)slot * w.seqs;
  fetch(n0);
  bool begun = false;
  for (; n0 < a.N; n0 += step) {
    bool odd = false;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      if (kseq[i] < w.seqs) {
        *reinterpret_cast<uint4*>(sk + kat[i]) = nk[i];
        *reinterpret_cast<uint4*>(sv + kat[i]) = nv[i];
        if (kat[i] % P == 0) there[kseq[i] * W + krow[i]] = nkeep >> i & 1;
        if constexpr (sizeof(E) == 2) odd = odd || Wide::odd(nk[i]) || Wide::odd(nv[i]);
        else odd = odd || Full::odd(nk[i]) || Full::odd(nv[i]);
      }
      if (qseq[i] < w.seqs) *reinterpret_cast<uint4*>(sq + qat[i]) = nq[i];
    }
    if (begun) leave(n0 - step);
    begun = true;
    bool some_odd = false;
    if (a.causal) some_odd = __syncthreads_or(odd);
    else __syncthreads();
    if ((int)threadIdx.x < w.seqs) lens[threadIdx.x] = nlen;      // for the outputs, after the last ones have gone
    if (n0 + step < a.N) fetch(n0 + step);
    for (int seq = 0, g = wave; ; g += 4) {
      while (g >= heads && seq < w.seqs) g -= heads, ++seq;
      const int64_t n = n0 + seq;
      if (seq >= w.seqs || n >= a.N) break;
      const int h = h0 + g, kc = (a.group == 1 ? g : h / a.group - y0) * a.d;
      const uint32_t keys = (uint32_t)__ballot(lane < a.Tk && there[seq * W + (lane & (W - 1))]);
      const int len = a.lengths ? min(max(uniform(a.lengths[n]), 0), a.Tk) : a.Tk;
      const bool all = keys == (uint32_t)((1ull << W) - 1);
      const E *uk = sk + seq * W * P + kc, *uv = sv + seq * W * P + kc, *uq = sq + seq * W * P + g * a.d;
      E* uo = so + seq * W * P + g * a.d;
      const float* table = add + g * 2 * W + W - 1 + col - 4 * sub;      // less a key's place
      Frag fk[NT][KS];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          fk[t][s] = Tl::rows(uk + t * 16 * P, P, s, lane);
          if (!whole && (16 * s + 4 * sub >= a.d || 16 * t + col >= a.Tk)) fk[t][s] = Tl::zero();
        }
      }
      bool slow = false;       // of this sequence and head: others keep their bits
      if (some_odd) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
#pragma unroll
          for (int s = 0; s < KS; ++s) slow = slow || (16 * s + 4 * sub < a.d && (Tl::odd(fk[t][s]) || Tl::odd(Tl::rows(uv + t * 16 * P, P, s, lane))));
        }
        slow = __any(slow);
      }
#pragma unroll
      for (int u = 0; u < NT; ++u) {
        if (16 * u >= a.Tq || at + 16 * u >= len) break;
        const int last = a.causal ? min(at + 16 * u + 15, len - 1) : len - 1;        // no query of this tile sees a later key
        Frag fq[KS];
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          fq[s] = Tl::rows(uq + u * 16 * P, P, s, lane);
          if (!whole && 16 * s + 4 * sub >= a.d) fq[s] = Tl::zero();
        }
        floatx4 x[NT];
        float top = -__builtin_inff();
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          if (16 * t > last) break;
          floatx4 b;
#pragma unroll
          for (int r = 0; r < 4; ++r) b[r] = table[16 * (u - t) - r];
          x[t] = (floatx4)(0.f);
#pragma unroll
          for (int s = 0; s < KS; ++s) x[t] = Tl::mma(fk[t][s], fq[s], x[t]);
#pragma unroll
          for (int r = 0; r < 4; ++r) x[t][r] = b[r] == -__builtin_inff() ? b[r] : fmaf(x[t][r], a.scale, b[r]);      // chosen, not added: a product may be infinite
          if (!all) {
            const uint32_t bits = keys >> (16 * t + 4 * sub);
#pragma unroll
            for (int r = 0; r < 4; ++r) x[t][r] = bits >> r & 1 ? x[t][r] : -__builtin_inff();
          }
#pragma unroll
          for (int r = 0; r < 4; ++r) top = fmaxf(top, x[t][r]);
        }
        top = column_max<4>(top);
        float l = 0.f;
        floatx4 o[DT];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) o[dt] = (floatx4)(0.f);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          if (16 * t > last) break;
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            x[t][r] = weight_of(x[t][r], top);
            l += x[t][r];
          }
          if (!slow) gather<Tl, DT>(o, uv + 16 * t * P, P, Packed<Tl>(x[t]), lane);
          else gather_seen<Tl, DT>(o, uv + 16 * t * P, P, Packed<Tl>(x[t]), lane, [](int) { return 0; }, [&](int c) { return at + 16 * u + c - 16 * t; });
        }
        l = column_sum<4>(l);
        const int i = 16 * u + col;
        if (i < a.Tq) {
          store_column<Tl, DT>(uo + i * P, o, l == 0.f ? 0.f : sizeof(E) == 2 ? __builtin_amdgcn_rcpf(l) : 1.f / l, a.d, lane);
          if (a.lse && sub == 0 && at + i < len) a.lse[(n * a.heads + h) * a.Tq + i] = log_sum(top, l);
        }
      }
    }
    __syncthreads();
  }
  if (begun) leave(n0 - step);
}

// ---------------------------------------------------------------------------------------------------- few queries
//
// Up to 16 queries (one: a new snapshot) against many keys.  Up to R = 2 rows, of heads that share a key head or of queries, on the vector unit: a key's row is
// read by LPK lanes, 16 bytes each, by each of the wave's 64 / LPK groups another key, four keys of a group at a time.  Every group has a
// softmax of its own, over its own keys; they are joined at the end, in the wave, in the workgroup, and by k_attn_join where the keys
// are split among workgroups.  Memory bounds it: 2000 sequences of up to 512 keys, 8 heads of 64, bf16 in 222 us, 4.7 TB/s.
template <int LPK>
__device__ __forceinline__ float lanes_sum(float x) {      // over LPK neighbouring lanes
  if constexpr (LPK >= 2) x += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0xB1, 0xf, 0xf, true));       // quad_perm 1 0 3 2
  if constexpr (LPK >= 4) x += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0x4E, 0xf, 0xf, true));       // quad_perm 2 3 0 1
  if constexpr (LPK >= 8) x += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0x141, 0xf, 0xf, true));      // row_half_mirror
  if constexpr (LPK >= 16) x += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(x), 0x140, 0xf, 0xf, true));     // row_mirror
  if constexpr (LPK >= 32) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  }
  return x;
}

template <class E, int LPK, int R>
__global__ __launch_bounds__(256) void k_attn_few(Args a) {
  constexpr int PER = ops::Elem<E>::kPer, KW = 64 / LPK, U = 4, STEP = 4 * KW * U;      // keys of a workgroup's step
  constexpr int ROOM = R * (LPK * PER + 2);
  __shared__ float joined[4][ROOM];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), c = (lane % LPK) * PER, g = lane / LPK;
  const int rows = a.group * a.Tq, blocks = (rows + R - 1) / R, kvs = a.heads / a.group;
  const uint32_t part = blockIdx.x % a.splits;
  uint32_t rest = blockIdx.x / a.splits;
  const int r0 = (int)(rest % blocks) * R;
  rest /= blocks;
  const int y = rest % kvs;
  const int64_t n = rest / kvs;
  const Seq q(a, n);
  float fq[R][PER], far[R];
  int p[R], most = -1, least = 0x7fffffff;
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int row = r0 + r, h = y * a.group + row / a.Tq, i = row % a.Tq;
    const bool live = row < rows && i >= q.lo && i < q.hi;
    p[r] = live ? (int)(q.at + i) : -1;
    if (live) most = max(most, p[r]), least = min(least, p[r]);
    uint4 w = make_uint4(0, 0, 0, 0);
    if (live && c < a.d) w = *reinterpret_cast<const uint4*>(static_cast<const E*>(a.q.p) + (int64_t)i * a.q.st + n * a.q.sn + h * a.d + c);
    ops::Elem<E>::unpack(w, fq[r]);
#pragma unroll
    for (int e = 0; e < PER; ++e) fq[r][e] *= a.scale;
    far[r] = a.bias && live ? bias_at(a, h, a.reach) : 0.f;
  }
  const int kend = most < 0 ? 0 : a.causal ? min(q.len, most + 1) : q.len;
  const int share = ((kend + a.splits - 1) / a.splits + STEP - 1) / STEP * STEP;
  const int k0 = (int)min((int64_t)part * share, (int64_t)kend), k1 = min(k0 + share, kend);
  const E* kbase = static_cast<const E*>(a.k.p) + n * a.k.sn + y * a.d + c;
  const E* vbase = static_cast<const E*>(a.v.p) + n * a.v.sn + y * a.d + c;
  float o[R][PER], m[R], l[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = -__builtin_inff();
    l[r] = 0.f;
#pragma unroll
    for (int e = 0; e < PER; ++e) o[r][e] = 0.f;
  }
  for (int j0 = k0 + wave * KW * U; j0 < k1; j0 += STEP) {
    uint4 wk[U], wv[U];
    bool in[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u * KW + g;
      in[u] = j < k1 && (!a.keep || a.keep[(int64_t)j * a.N + n]);
      const bool ok = in[u] && c < a.d;
      wk[u] = ok ? *reinterpret_cast<const uint4*>(kbase + (int64_t)j * a.k.st) : make_uint4(0, 0, 0, 0);
      wv[u] = ok ? *reinterpret_cast<const uint4*>(vbase + (int64_t)j * a.v.st) : make_uint4(0, 0, 0, 0);
    }
    const bool near = a.bias && least - (j0 + KW * U - 1) < a.reach;
    const bool edge = a.causal && j0 + KW * U - 1 > least;       // not every row sees every key
    float x[R][U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float k[PER];
      ops::Elem<E>::unpack(wk[u], k);
      const int j = j0 + u * KW + g;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float s = fq[r][0] * k[0];
#pragma unroll
        for (int e = 1; e < PER; ++e) s = fmaf(fq[r][e], k[e], s);
        s = lanes_sum<LPK>(s);
        if (near) s += bias_at(a, y * a.group + min(r0 + r, rows - 1) / a.Tq, (int64_t)p[r] - j);
        else s += far[r];
        x[r][u] = in[u] && p[r] >= 0 && (!edge || j <= p[r]) ? s : -__builtin_inff();
      }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float top = m[r];
#pragma unroll
      for (int u = 0; u < U; ++u) top = fmaxf(top, x[r][u]);
      const float keepf = weight_of(m[r], top);
      m[r] = top;
      l[r] *= keepf;
#pragma unroll
      for (int e = 0; e < PER; ++e) o[r][e] *= keepf;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const bool out = edge && x[r][u] == -__builtin_inff();     // unseen: its values do not count, whatever they are
        x[r][u] = weight_of(x[r][u], top);
        l[r] += x[r][u];
        float v[PER];
        ops::Elem<E>::unpack(out ? make_uint4(0, 0, 0, 0) : wv[u], v);
#pragma unroll
        for (int e = 0; e < PER; ++e) o[r][e] = fmaf(x[r][u], v[e], o[r][e]);
      }
    }
  }
  // The groups of a wave, then the waves.
#pragma unroll
  for (int r = 0; r < R; ++r) {
    float top = m[r];
    for (int s = LPK; s < 64; s *= 2) top = fmaxf(top, __shfl_xor(top, s));
    const float f = weight_of(m[r], top);
    m[r] = top;
    l[r] *= f;
    for (int s = LPK; s < 64; s *= 2) l[r] += __shfl_xor(l[r], s);
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      o[r][e] *= f;
      for (int s = LPK; s < 64; s *= 2) o[r][e] += __shfl_xor(o[r][e], s);
    }
    if (g == 0) {
      float* to = joined[wave] + r * (LPK * PER + 2);
#pragma unroll
      for (int e = 0; e < PER; ++e) to[c + e] = o[r][e];
      if (c == 0) to[LPK * PER] = m[r], to[LPK * PER + 1] = l[r];
    }
  }
  __syncthreads();
  for (int r = wave; r < R; r += 4) {
    const int row = r0 + r;
    if (row >= rows) continue;
    const int h = y * a.group + row / a.Tq, i = row % a.Tq;
    if (i < q.lo || i >= q.hi) continue;
    float top = -__builtin_inff(), f[4], sum = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, joined[w][r * (LPK * PER + 2) + LPK * PER]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      f[w] = weight_of(joined[w][r * (LPK * PER + 2) + LPK * PER], top);
      sum = fmaf(joined[w][r * (LPK * PER + 2) + LPK * PER + 1], f[w], sum);
    }
    const int64_t at = (n * a.heads + h) * a.Tq + i;
    const float by = a.splits > 1 ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
    for (int e = lane; e < a.d; e += 64) {
      float v = 0.f;
#pragma unroll
      for (int w = 0; w < 4; ++w) v = fmaf(joined[w][r * (LPK * PER + 2) + e], f[w], v);
      v *= by;
      if (a.splits > 1) a.joint[(at * a.splits + part) * (a.d + 2) + e] = v;
      else static_cast<E*>(const_cast<void*>(a.o.p))[(int64_t)i * a.o.st + n * a.o.sn + h * a.d + e] = ops::Elem<E>::one(v);
    }
    if (lane == 0) {
      if (a.splits > 1) {
        a.joint[(at * a.splits + part) * (a.d + 2) + a.d] = top;
        a.joint[(at * a.splits + part) * (a.d + 2) + a.d + 1] = sum;
      } else if (a.lse) {
        a.lse[at] = log_sum(top, sum);
      }
    }
  }
}

// More rows than two, of heads that share a key head or of several queries: 16 of them are the columns of a matrix product, so a key is read once for
// all (two sequences of 65 536 keys, 4 key heads of 128 for 16, bf16: 66 us, of which 55 at a copy's rate; two rows at a time on the vector unit 240; fp32: 114 us, 4.7 TB/s).  A wave takes 32 keys at a time (16 of wide fp32 rows): their rows go from memory into operands, values through LDS (each wave's own part), four waves a workgroup.
template <class E> struct Slab;
template <> struct Slab<uint16_t> {
  static constexpr int PER = 8, STEP = 32;      // elements of a lane, contraction of a product
  static __device__ __forceinline__ floatx4 mma(uint4 a, uint4 b, floatx4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  // o += values^T weights for 32 keys: element e of a lane stands for key 4 sub + e of the first 16, then of the second.
  template <int DT, int NT>
  static __device__ __forceinline__ void add(floatx4 (&o)[DT], const uint16_t* sv, int pitch, const floatx4 (&x)[NT], int lane) {
    const uint4 b = make_uint4(pack2(x[0][0], x[0][1]), pack2(x[0][2], x[0][3]), pack2(x[1][0], x[1][1]), pack2(x[1][2], x[1][3]));
    const uint16_t* at = sv + (4 * (lane >> 4) + ((lane & 15) >> 2)) * pitch + 4 * (lane & 3);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const uint2 u = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4)(at + 16 * dt)));
      const uint2 w = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_shortx4)(at + 16 * pitch + 16 * dt)));
      o[dt] = mma(make_uint4(u.x, u.y, w.x, w.y), b, o[dt]);
    }
  }
  static __device__ __forceinline__ bool odd(uint4 w) { return Wide::odd(w); }
  static __device__ __forceinline__ float get(const uint16_t* p) { return __uint_as_float((uint32_t)*p << 16); }
};
template <> struct Slab<float> {
  static constexpr int PER = 4, STEP = 16;
  static __device__ __forceinline__ floatx4 mma(uint4 a, uint4 b, floatx4 c) { return Full::mma(a, b, c); }
  template <int DT, int NT>
  static __device__ __forceinline__ void add(floatx4 (&o)[DT], const float* sv, int pitch, const floatx4 (&x)[NT], int lane) {
#pragma unroll
    for (int t = 0; t < NT; ++t) gather<Full, DT>(o, sv + 16 * t * pitch, pitch, Packed<Full>(x[t]), lane);
  }
  static __device__ __forceinline__ bool odd(uint4 w) { return Full::odd(w); }
  static __device__ __forceinline__ float get(const float* p) { return *p; }
};

template <class E, int D>
__global__ __launch_bounds__(256, 2) void k_attn_rows(Args a) {
  typedef Slab<E> S;
  constexpr int NT = sizeof(E) * D > 256 ? 1 : 2, KEYS = 16 * NT;      // of a step, as registers allow
  constexpr int KS = D / S::STEP, DT = D / 16, P = D + 16 / (int)sizeof(E), ROW = D + 2;
  constexpr int VALUES = 4 * KEYS * P * (int)sizeof(E), JOINED = 4 * 16 * ROW * 4;
  __shared__ __attribute__((aligned(16))) char room[VALUES > JOINED ? VALUES : JOINED];
  __shared__ float weights[4][KEYS][17];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6), col = lane & 15, sub = lane >> 4;
  const int rows = a.group * a.Tq, blocks = (rows + 15) / 16, kvs = a.heads / a.group;
  const uint32_t part = blockIdx.x % a.splits;
  uint32_t rest = blockIdx.x / a.splits;
  const int r0 = (int)(rest % blocks) * 16;
  rest /= blocks;
  const int y = rest % kvs;
  const int64_t n = rest / kvs;
  const Seq q(a, n);
  E* const sv = reinterpret_cast<E*>(room) + wave * KEYS * P;
  const int row = r0 + col, h = y * a.group + min(row, rows - 1) / a.Tq, i = row % a.Tq;
  const bool live = row < rows && i >= q.lo && i < q.hi;
  const int p = live ? (int)(q.at + i) : -1;
  int most = p, least = live ? p : 0x7fffffff;
#pragma unroll
  for (int m = 1; m < 16; m *= 2) most = max(most, __shfl_xor(most, m)), least = min(least, __shfl_xor(least, m));
  most = uniform(most);
  least = uniform(least);
  uint4 fq[KS];
  const E* qrow = static_cast<const E*>(a.q.p) + (int64_t)i * a.q.st + n * a.q.sn + h * a.d;
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    const int c = S::STEP * s + S::PER * sub;
    fq[s] = live && c < a.d ? *reinterpret_cast<const uint4*>(qrow + c) : make_uint4(0, 0, 0, 0);
  }
  const float far = a.bias ? bias_at(a, h, a.reach) : 0.f;
  const int kend = most < 0 ? 0 : a.causal ? min(q.len, most + 1) : q.len;
  const int share = ((kend + a.splits - 1) / a.splits + 127) / 128 * 128;
  const int k0 = (int)min((int64_t)part * share, (int64_t)kend), k1 = min(k0 + share, kend);
  const E* kbase = static_cast<const E*>(a.k.p) + n * a.k.sn + y * a.d + S::PER * sub;
  const E* vbase = static_cast<const E*>(a.v.p) + n * a.v.sn + y * a.d + S::PER * sub;
  floatx4 o[DT];
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) o[dt] = (floatx4)(0.f);
  float m = -__builtin_inff(), l = 0.f;
  uint4 wk[NT][KS], wv[NT][KS];
  uint32_t bits = 0;         // which of the step's keys are there
  auto fetch = [&](int j0) __attribute__((always_inline)) {
    const int mine = j0 + (lane & (KEYS - 1));
    bits = (uint32_t)__ballot(mine < k1 && (!a.keep || a.keep[(int64_t)mine * a.N + n]));
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int j = j0 + 16 * t + col;
      const bool in = bits >> (16 * t + col) & 1;
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        const bool ok = in && S::STEP * s + S::PER * sub < a.d;
        wk[t][s] = ok ? *reinterpret_cast<const uint4*>(kbase + (int64_t)j * a.k.st + S::STEP * s) : make_uint4(0, 0, 0, 0);
        wv[t][s] = ok ? *reinterpret_cast<const uint4*>(vbase + (int64_t)j * a.v.st + S::STEP * s) : make_uint4(0, 0, 0, 0);
      }
    }
  };
  int j0 = k0 + wave * KEYS;
  if (j0 < k1) fetch(j0);
  for (; j0 < k1; j0 += 4 * KEYS) {
    wave_fence();
    bool bad = false;
    floatx4 x[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      x[t] = (floatx4)(0.f);
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        x[t] = S::mma(wk[t][s], fq[s], x[t]);
        bad = bad || S::odd(wv[t][s]);
        *reinterpret_cast<uint4*>(sv + (16 * t + col) * P + S::STEP * s + S::PER * sub) = wv[t][s];
      }
    }
    const uint32_t there = bits;
    if (j0 + 4 * KEYS < k1) fetch(j0 + 4 * KEYS);
    const bool near = a.bias && least - (j0 + KEYS - 1) < a.reach, edge = a.causal && j0 + KEYS - 1 > least;
    float top = m;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int at = 16 * t + 4 * sub + r;
        const float b = near ? bias_at(a, h, (int64_t)p - (j0 + at)) : far;
        x[t][r] = live && (there >> at & 1) && (!edge || j0 + at <= p) ? fmaf(x[t][r], a.scale, b) : -__builtin_inff();
        top = fmaxf(top, x[t][r]);
      }
    }
    top = column_max<4>(top);
    const float f = weight_of(m, top);
    m = top;
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        x[t][r] = weight_of(x[t][r], top);
        sum += x[t][r];
      }
    }
    l = fmaf(l, f, sum);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] *= f;
    wave_fence();
    if (!edge || !__any(bad)) {
      S::add(o, sv, P, x, lane);
    } else {      // a zero weight would meet a value that is not finite: key by key, only where it is seen
#pragma unroll
      for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int r = 0; r < 4; ++r) weights[wave][16 * t + 4 * sub + r][col] = x[t][r];
      }
      wave_fence();
#pragma unroll 1
      for (int at = 0; at < KEYS; ++at) {
        const bool seen = j0 + at <= p;
        const float w = weights[wave][at][col];
#pragma unroll
        for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float v = seen ? S::get(sv + at * P + 16 * dt + 4 * sub + r) : 0.f;
            o[dt][r] = fmaf(w, v, o[dt][r]);
          }
        }
      }
    }
  }
  l = column_sum<4>(l);
  // The waves' parts: a row's D sums, its maximum and its sum.
  __syncthreads();
  float* const joined = reinterpret_cast<float*>(room);
  float* to = joined + (wave * 16 + col) * ROW;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
#pragma unroll
    for (int r = 0; r < 4; ++r) to[16 * dt + 4 * sub + r] = o[dt][r];
  }
  if (sub == 0) to[D] = m, to[D + 1] = l;
  __syncthreads();
  const int mine = threadIdx.x >> 4, r = r0 + mine, hm = y * a.group + min(r, rows - 1) / a.Tq, im = r % a.Tq;
  if (r >= rows || im < q.lo || im >= q.hi) return;
  float top = -__builtin_inff(), f[4], sum = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) top = fmaxf(top, joined[(w * 16 + mine) * ROW + D]);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    f[w] = weight_of(joined[(w * 16 + mine) * ROW + D], top);
    sum = fmaf(joined[(w * 16 + mine) * ROW + D + 1], f[w], sum);
  }
  const int64_t at = (n * a.heads + hm) * a.Tq + im;
  const float by = a.splits > 1 ? 1.f : sum == 0.f ? 0.f : 1.f / sum;
  for (int e = threadIdx.x & 15; e < a.d; e += 16) {
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) v = fmaf(joined[(w * 16 + mine) * ROW + e], f[w], v);
    v *= by;
    if (a.splits > 1) a.joint[(at * a.splits + part) * (a.d + 2) + e] = v;
    else static_cast<E*>(const_cast<void*>(a.o.p))[(int64_t)im * a.o.st + n * a.o.sn + hm * a.d + e] = ops::Elem<E>::one(v);
  }
  if ((threadIdx.x & 15) == 0) {
    if (a.splits > 1) {
      a.joint[(at * a.splits + part) * (a.d + 2) + a.d] = top;
      a.joint[(at * a.splits + part) * (a.d + 2) + a.d + 1] = sum;
    } else if (a.lse) {
      a.lse[at] = log_sum(top, sum);
    }
  }
}

// The parts of split keys: a workgroup a row, two elements a lane, a quarter of the parts a wave.
template <class E>
__global__ __launch_bounds__(256) void k_attn_join(Args a) {
  __shared__ float factor[kMaxSplits], tops[4], sums[4], joined[4][kMaxDim];
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int64_t at = blockIdx.x;
  const int i = (int)(at % a.Tq), h = (int)(at / a.Tq % a.heads);
  const int64_t n = at / a.Tq / a.heads;
  const Seq q(a, n);
  if (i < q.lo || i >= q.hi) return;
  const float* from = a.joint + at * a.splits * (a.d + 2);
  float top = -__builtin_inff();
  for (int s = threadIdx.x; s < a.splits; s += 256) top = fmaxf(top, from[s * (a.d + 2) + a.d]);
  for (int x = 1; x < 64; x *= 2) top = fmaxf(top, __shfl_xor(top, x));
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  float sum = 0.f;
  for (int s = threadIdx.x; s < a.splits; s += 256) {
    factor[s] = weight_of(from[s * (a.d + 2) + a.d], top);
    sum = fmaf(from[s * (a.d + 2) + a.d + 1], factor[s], sum);
  }
  sum = wave_sum(sum);
  if (lane == 0) sums[wave] = sum;
  __syncthreads();
  sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
  float v[2] = {0.f, 0.f};
  const int e = 2 * lane;
  if (e < a.d) {
#pragma unroll 8
    for (int s = wave; s < a.splits; s += 4) {
      const float2 u = *reinterpret_cast<const float2*>(from + s * (a.d + 2) + e);
      v[0] = fmaf(u.x, factor[s], v[0]);
      v[1] = fmaf(u.y, factor[s], v[1]);
    }
    joined[wave][e] = v[0];
    joined[wave][e + 1] = v[1];
  }
  __syncthreads();
  if ((int)threadIdx.x < a.d) {
    const float x = (joined[0][threadIdx.x] + joined[1][threadIdx.x]) + (joined[2][threadIdx.x] + joined[3][threadIdx.x]);
    static_cast<E*>(const_cast<void*>(a.o.p))[(int64_t)i * a.o.st + n * a.o.sn + h * a.d + threadIdx.x] = ops::Elem<E>::one(sum == 0.f ? 0.f : x / sum);
  }
  if (a.lse && threadIdx.x == 0) a.lse[at] = log_sum(top, sum);
}

// ---------------------------------------------------------------------------------------------------- choice and launch

template <class Tl, int NT>
void window(Args a, hipStream_t st) {
  const int64_t waves = 256 * 32;      // as many as the card holds at a time
  a.slots = (int)std::min<int64_t>(a.N, (waves + a.heads - 1) / a.heads);
  const unsigned grid = (unsigned)(((int64_t)a.slots * a.heads + 3) / 4);
  if constexpr (NT <= 2) {
    const int e = sizeof(typename Tl::E), W = 16 * NT;
    auto far = [&](const Rows& x) { return (x.st > x.sn ? x.st : x.sn) >= ((int64_t)1 << 31) / e / (W + 2); };      // beyond 32-bit offsets
    if (!a.first && !far(a.k) && !far(a.v) && !far(a.q) && !far(a.o)) {
      WindowArgs w{a};
      w.together = std::min(a.heads, std::max(1, 256 / (a.d * e)));
      w.seqs = w.together >= 4 || a.d * e > 256 ? 1 : 2;
      w.groups = (a.heads + w.together - 1) / w.together;
      w.pitch = w.together * a.d + 16 / e;
      const int64_t blocks = (a.N + w.seqs - 1) / w.seqs, most = 256 * 8;
      w.a.slots = (int)std::min<int64_t>(blocks, (most + w.groups - 1) / w.groups);
      const unsigned lds = 4 * w.seqs * W * w.pitch * e + 64 * e + 4 * (w.together * 2 * W + w.seqs * W + w.seqs), wgs = (unsigned)(w.a.slots * w.groups);
      const bool more = w.seqs * W * std::max(1, w.together * a.d * e / 16) > 256 * NT;
#define DGC_WINDOWS(KS)                                                                                  \
  if (more) hipLaunchKernelGGL((k_attn_windows<Tl, NT, KS, 2 * NT>), wgs, 256, lds, st, w);    \
  else hipLaunchKernelGGL((k_attn_windows<Tl, NT, KS, NT>), wgs, 256, lds, st, w)
      if (lds > 65536) {
        // below
      } else if (a.d <= 16) {
        DGC_WINDOWS(1);
      } else if (a.d <= 32) {
        DGC_WINDOWS(2);
      } else if (a.d <= 64) {
        DGC_WINDOWS(4);
      } else {
        DGC_WINDOWS(8);
      }
#undef DGC_WINDOWS
      if (lds <= 65536) return;
    }
  }
  if (a.d <= 16) hipLaunchKernelGGL((k_attn_window<Tl, NT, 1>), grid, 256, 0, st, a);
  else if (a.d <= 32) hipLaunchKernelGGL((k_attn_window<Tl, NT, 2>), grid, 256, 0, st, a);
  else if (a.d <= 64) hipLaunchKernelGGL((k_attn_window<Tl, NT, 4>), grid, 256, 0, st, a);
  else hipLaunchKernelGGL((k_attn_window<Tl, NT, 8>), grid, 256, 0, st, a);
}

template <class E, int D>
void few_rows(const Args& a, unsigned grid, hipStream_t st) {
  constexpr int LPK = D / ops::Elem<E>::kPer;
  const int rows = a.group * a.Tq;
  if (rows == 1) hipLaunchKernelGGL((k_attn_few<E, LPK, 1>), grid, 256, 0, st, a);
  else if (rows == 2) hipLaunchKernelGGL((k_attn_few<E, LPK, 2>), grid, 256, 0, st, a);
  else hipLaunchKernelGGL((k_attn_rows<E, (D > 16 || sizeof(E) == 4 ? D : 32)>), grid, 256, 0, st, a);
}
template <class E>
void few(const Args& a, hipStream_t st) {
  const int64_t rows = (int64_t)a.group * a.Tq;
  const unsigned grid = (unsigned)(a.N * (a.heads / a.group) * ((rows + 15) / 16) * a.splits);
  if (a.d <= 16) few_rows<E, 16>(a, grid, st);
  else if (a.d <= 32) few_rows<E, 32>(a, grid, st);
  else if (a.d <= 64) few_rows<E, 64>(a, grid, st);
  else few_rows<E, 128>(a, grid, st);
  if (a.splits > 1) hipLaunchKernelGGL(k_attn_join<E>, (unsigned)(a.N * a.heads * a.Tq), 256, 0, st, a);
}
// fp32 heads go in steps of 16 or 32 columns, where 40 x 512 tokens, 8 heads of 96 take 196 us with 96 and 245 with 128 columns, 8 of 40 107 with 48 and 116 with 64.
template <class Tl>
void large(const Args& a, hipStream_t st) {
  const unsigned grid = (unsigned)(a.N * a.heads * ((a.Tq + 4 * Tl::M - 1) / (4 * Tl::M)));
  const unsigned lds = bias_bytes(a);
  if (a.d <= 16) hipLaunchKernelGGL((k_attn_forward<Tl, 1>), grid, 256, lds, st, a);
  else if (a.d <= 32) hipLaunchKernelGGL((k_attn_forward<Tl, 2>), grid, 256, lds, st, a);
  else if (a.d <= 48 && Tl::kExact) hipLaunchKernelGGL((k_attn_forward<Tl, Tl::kExact ? 3 : 4>), grid, 256, lds, st, a);
  else if (a.d <= 64) hipLaunchKernelGGL((k_attn_forward<Tl, 4>), grid, 256, lds, st, a);
  else if (a.d <= 96 && Tl::kExact) hipLaunchKernelGGL((k_attn_forward<Tl, Tl::kExact ? 6 : 8>), grid, 256, lds, st, a);
  else hipLaunchKernelGGL((k_attn_forward<Tl, 8>), grid, 256, lds, st, a);
}

template <class Tl16, class TlLong>
void forward(const Args& a, hipStream_t st) {
  switch (form_of(a.Tq, a.Tk)) {
    case kWindow:
      if (a.Tk <= 16) window<Tl16, 1>(a, st);
      else if (a.Tk <= 32) window<Tl16, 2>(a, st);
      else window<Tl16, 4>(a, st);
      break;
    case kFew: few<typename Tl16::E>(a, st); break;
    default: large<TlLong>(a, st);
  }
}

}  // namespace

void attn_forward_f32(const Args& a, hipStream_t st) { forward<Full, Full>(a, st); }
void attn_forward_bf16(const Args& a, hipStream_t st) { forward<Small, Wide>(a, st); }

}  // namespace attn
}  // namespace dgc
