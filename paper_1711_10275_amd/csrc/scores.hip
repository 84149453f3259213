// What a per-site classifier answers with and learns from: per active site
// the log probability of its label, the entropy of its class distribution and
// the best classes, and the gradient of those numbers at the logits.
//
// Row x of `classes` values, m = max x, t = sum of exp(x_k - m) over all
// classes but one largest, L = log1p(t) (so log sum exp x = m + L):
//   log p_k = (x_k - m) - L,   H = L - sum_k exp(x_k - m) (x_k - m) / (1 + t).
// Leaving the largest (a 1) out of t keeps a sure row's small numbers: its
// log probability is -t, where log(1 + t) would have dropped t's low bits.
// Sums are fp32, over the values as they are stored.
#include <algorithm>
#include <type_traits>

#include "internal.h"
#include "numeric.h"
#include "wave.h"

namespace sscn {

namespace {

constexpr int kMaxTop = 16;  // best classes a call may ask for

// Order of the best classes as one whole number, larger first: by value (NaN
// above everything, -0 equal to 0), ties to the lowest class.
__device__ __forceinline__ uint64_t rank_key(float x, uint32_t cls) {
  const uint32_t b = __float_as_uint(x + 0.f);
  const uint32_t o = x != x ? 0xfffffffeu : ((int32_t)b < 0 ? ~b : b | 0x80000000u);
  return (uint64_t)o << 32 | (0xffffffffu - cls);
}
__device__ __forceinline__ uint32_t key_class(uint64_t k) { return 0xffffffffu - (uint32_t)k; }
__device__ __forceinline__ float key_value(uint64_t k) {  // NaN for NaN, 0 for -0
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float((int32_t)o < 0 ? o & 0x7fffffffu : ~o);
}

// ------------------------------------------------------------- longer rows
// A team of L lanes (L = 16 or 64: within one wavefront; L = 256: a workgroup)
// holds a chunk of up to L E values of a row in registers as they are stored:
// one read of the logits, the maximum before the exponentials.  Lanes take
// 16-byte pieces of V values, from the row's start on and at whatever alignment
// that has (the hardware takes any).  A piece that the row's end cuts is the
// row's last V values, of which those of the piece before are made -inf; so is
// all of a piece beyond the end.
template <typename T, int L, int E>
struct Chunk {
  static constexpr int V = 16 / (int)sizeof(T);  // values per piece
  static constexpr int G = E / V;                // pieces per lane
  static constexpr int kSpan = L * V;            // values of the team's g-th pieces
  static constexpr int kValues = L * E;

  uint32_t w[G][4];  // bf16 two to a word
  // Lane of the team; values of the chunk, at most kValues.  (A chunk of fewer
  // than V is a row's last, and its one piece starts in the chunk before.)
  int lane, len;

  // Whether the g-th pieces hold anything: the same for the whole team.
  __device__ bool has(int g) const { return g * kSpan < len; }
  // Place in the chunk of this lane's piece g.
  __device__ int place(int g) const { return min((g * L + lane) * V, len - V); }
  __device__ float at(int g, int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[g][i]);
    else return __uint_as_float(i % 2 ? w[g][i / 2] & 0xffff0000u : w[g][i / 2] << 16);
  }
  __device__ void load(const T* p, int lane_, int len_) {
    lane = lane_;
    len = len_;
    // Each turn forms the places and masks below anew: kept over the row loop
    // they took 70 more registers, and half of the wavefronts that fit.
    asm volatile("" : "+v"(lane), "+s"(len));
#pragma unroll
    for (int g = 0; g < G; ++g)
      if (has(g)) __builtin_memcpy(w[g], p + place(g), 16);
#pragma unroll
    for (int g = 0; g < G; ++g)
      if (has(g) && (g + 1) * kSpan > len) {
        const int twice = (g * L + lane) * V - place(g);  // values that the pieces before have
#pragma unroll
        for (int i = 0; i < V; ++i)
          if constexpr (sizeof(T) == 4) {
            w[g][i] = i < twice ? 0xff800000u : w[g][i];  // -inf
          } else {
            const uint32_t none = i % 2 ? 0xff800000u : 0xff80u, rest = i % 2 ? 0xffffu : 0xffff0000u;
            w[g][i / 2] = i < twice ? (w[g][i / 2] & rest) | none : w[g][i / 2];
          }
      }
  }
};

// What one chunk (or several joined) says of a row: m, t = sum of exp(x - m)
// but one largest, a = sum of exp(x - m) (x - m).
struct Part {
  float m, t, a;
};
__device__ __forceinline__ Part join(const Part& p, const Part& q) {
  const bool first = p.m >= q.m;
  const Part &hi = first ? p : q, &lo = first ? q : p;
  if (lo.m == -INFINITY) return {OpMax::of(p.m, q.m), hi.t, hi.a};
  const float d = lo.m - hi.m, e = expf(d);
  // the low part's values, its largest among them, shift by d
  return {OpMax::of(p.m, q.m), hi.t + e * (1.f + lo.t), hi.a + e * (lo.a + (d < -200.f ? -200.f : d) * (1.f + lo.t))};
}
// log(1 + t), t >= 0: log(u) t / (u - 1) for u = 1 + t as rounded, in which
// u's rounding cancels (Goldberg, "What every computer scientist should know
// about floating-point arithmetic", theorem 4).  Good to 6 half steps.
__device__ __forceinline__ float log_1p(float t) {
  const float u = 1.f + t;
  return u == 1.f ? t : __builtin_amdgcn_logf(u) * 0.69314718055994530942f * (t * __builtin_amdgcn_rcpf(u - 1.f));
}
__device__ __forceinline__ float2 finish(const Part& p) {
  if (p.m == INFINITY || p.m != p.m) return make_float2(NAN, NAN);
  if (p.m == -INFINITY) return make_float2(0.f, 0.f);
  const float l = log_1p(p.t);
  return make_float2(l, l - p.a * __builtin_amdgcn_rcpf(1.f + p.t));
}

// Sums of e^(x - m) and e^(x - m) (x - m) as powers of two, h = (x - m) log2(e).
// h is one rounded product: a term is off by up to 2.25 |x - m| half steps,
// which its own size e^(x - m) outweighs; forming the product's low part too
// would cost three more operations a value.  Below 2^-126 the power of two is 0.
struct ExpSums {
  float base, s = 0.f, a = 0.f;
  __device__ explicit ExpSums(float m) : base(m == -INFINITY ? 0.f : m) {}
  __device__ __forceinline__ void add(float x) {
    const float h = fmaxf((x - base) * 1.44269504088896340736f, -300.f);  // 2^-300 is 0: no 0 * inf
    const float e = __builtin_amdgcn_exp2f(h);
    s += e;
    a = fmaf(e, h, a);
  }
};

struct Outputs {
  float *logprob, *entropy, *stats;
  int32_t* top_index;
  float* top_logprob;
};
// A row's label and its logit, read before the row's work.
struct Label {
  int k;
  float x;
};
template <typename T>
__device__ __forceinline__ Label label_of(const T* row, const int32_t* labels, int64_t r, int classes) {
  const int k = labels ? labels[r] : -1;
  return {k, k >= 0 && k < classes ? ld(row + k) : k < 0 ? 0.f : NAN};
}

// Writes row r, by lanes 0 .. 15 of a team.  top: top_k keys in LDS, best
// first, 0 where the row has fewer classes above -inf: the lowest of the
// others follow.
__device__ __forceinline__ void write_row(int lane, int64_t r, const Label& lab, int top_k, const Part& p,
                                          uint64_t* top, const Outputs& o) {
  const float2 lh = finish(p);
  const float base = p.m == -INFINITY ? 0.f : p.m;
  if (top_k > 0 && lane == 0 && top[top_k - 1] == 0) {
    int have = 0;
    while (top[have] != 0) ++have;
    uint32_t k = 0;
    for (int j = have; j < top_k; ++k) {
      bool listed = false;
      for (int i = 0; i < have; ++i) listed |= key_class(top[i]) == k;
      if (!listed) top[j++] = rank_key(-INFINITY, k);
    }
  }
  if (lane == 0) {
    if (o.logprob) o.logprob[r] = lab.k < 0 ? 0.f : (lab.x - base) - lh.x;
    o.entropy[r] = lh.y;
    reinterpret_cast<float2*>(o.stats)[r] = make_float2(p.m, lh.x);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (lane < top_k) {
    const uint64_t key = top[lane];
    o.top_index[r * top_k + lane] = (int32_t)key_class(key);
    o.top_logprob[r * top_k + lane] = (key_value(key) - base) - lh.x;
  }
}

// The k-th largest of the 32 values v0, v1 of the 16 lanes of each row.
__device__ __forceinline__ float kth_of_32(float v0, float v1, int k) {
  const float hi = fmaxf(v0, v1), lo = fminf(v0, v1);
  const int above_hi = above_in_row(hi, hi) + above_in_row(lo, hi);
  const int above_lo = above_in_row(hi, lo) + above_in_row(lo, lo) + (hi > lo);
  return wave_reduce<OpMin, 1, 16>(above_lo < k ? lo : above_hi < k ? hi : INFINITY);
}

// Teams of W wavefronts (W = 1: 64 / L teams to a workgroup of one wavefront,
// a whole row each; W = 4: L = 64 lanes of each wavefront together, one chunk
// of one row, blockIdx.x the chunk).  Where a row is one chunk it is written,
// else its Part and its best keys are left for k_scores_join.
//
// The best classes: T, the least of at least top_k groups' maxima (groups of
// lanes that share no value), is no larger than the top_k-th best value, so
// what is below T is out.  Few values are left (about top_k log(top_k) of
// unordered ones); each counts the keys above its own, which is its rank.
// Values of -inf stay out of the list.  Masks that leave some group nothing
// make T -inf: the largest is taken off a long list top_k times.  A list that
// overflows (ties at T), or a NaN, takes them off the row itself.
// KT: at most as many best classes (0, 8 or 16: what fewer need takes fewer
// registers).
//
// 4096 x 40001 bf16 (328 MB, 60 us at the card's copy rate): 64 us without best
// classes, memory-bound (10.5 issue slots a value for unpacking, maximum and sums
// are 44 us of the vector units, behind other workgroups' loads), and the join's
// 5; with the best 8, whose listing and ranking is work on top, 87 and 8.
// (Keeping the chunk packed and the rare ways out of the registers took 124
// registers to 70 and 185 us to 113; the threshold from 16 groups 108 to 97.)
// Many equal logits at the threshold overflow the list, and the best classes come
// off the row one by one: with all logits equal, best 8, 300,000 x 200 bf16 take
// 422 us for 107, 4096 x 40001 1070 for 93.
template <typename T, int L, int W, int E, int KT>
__global__ __launch_bounds__(64 * W) void k_scores_chunk(const T* __restrict__ z, int64_t ldz, int64_t n, int classes,
                                                         const int32_t* __restrict__ labels, int top_k, Outputs o,
                                                         float4* __restrict__ part_out,
                                                         uint64_t* __restrict__ keys_out) {
  using C = Chunk<T, L * W, E>;
  constexpr int kTeams = 64 / L;  // to a wavefront
  // keys that a wavefront's part of a team may list, and may rank
  constexpr int kList = L == 16 ? 128 : L * E < 512 ? L * E : 512, kRanked = 128 / W;
  __shared__ uint64_t lists[kTeams * W][kList], tops[kTeams][kMaxTop], most[2][W];
  __shared__ float red[8 * W], sums[3][W];
  __shared__ int counts[W];
  static_assert(W == 1 || (W == 4 && L == 64));
  const int wave = threadIdx.x >> 6;
  const int team = (threadIdx.x & 63) / L, lane = threadIdx.x & (L - 1);  // lane of the team's part of this wavefront
  const int all = W == 1 ? lane : (int)threadIdx.x;                       // lane of the team
  uint64_t *list = lists[W == 1 ? team : wave], *top = tops[team];
  const int parts = W == 1 ? 1 : (int)gridDim.x;
  const int64_t rows = W == 1 ? (int64_t)gridDim.x * kTeams : gridDim.y;
  for (int64_t r0 = W == 1 ? (int64_t)blockIdx.x * kTeams : blockIdx.y; r0 < n; r0 += rows) {
    const int64_t r = min<int64_t>(r0 + team, n - 1);
    const bool live = r0 + team < n;  // a last team without a row works on the last one, and does not write
    const T* row = z + r * ldz;
    const int k0 = W == 1 ? 0 : (int)blockIdx.x * C::kValues;
    C x;
    x.load(row + k0, all, min(classes - k0, C::kValues));
    Label lab{-1, 0.f};
    if (wave == 0 && lane == 0) lab = label_of(row, labels, r, classes);
    // this lane's maxima: of its pieces, of all their first and second halves
    float piece[C::G], half0 = -INFINITY, half1 = -INFINITY;
#pragma unroll
    for (int g = 0; g < C::G; ++g) {
      piece[g] = -INFINITY;
      if (!x.has(g)) continue;
      float m0 = x.at(g, 0), m1 = x.at(g, C::V / 2);
#pragma unroll
      for (int i = 1; i < C::V / 2; ++i) {
        m0 = OpMax::of(m0, x.at(g, i));
        m1 = OpMax::of(m1, x.at(g, C::V / 2 + i));
      }
      piece[g] = OpMax::of(m0, m1);
      half0 = OpMax::of(half0, m0);
      half1 = OpMax::of(half1, m1);
    }
    const float own = OpMax::of(half0, half1);
    // the threshold: the top_k-th largest of 16 maxima, of 32 for more than 8
    // (lanes or their halves, of four wavefronts rows of lanes or their halves; of
    // one wavefront the least of its four rows' top_k / 4-th largest)
    float m = W == 1 ? wave_reduce<OpMax, 1, L>(own) : 0.f, cut = m;
    if constexpr (KT == 0) {
    } else if constexpr (L == 16) {
      if (KT > 8 && top_k > 8) {
        cut = kth_of_32(half0, half1, top_k);
      } else if (top_k > 1) {
        cut = wave_reduce<OpMin, 1, 16>(above_in_row(own, own) < top_k ? own : INFINITY);
      }
    } else if constexpr (W == 1) {
      if (top_k > 1) cut = wave_reduce<OpMin>(above_in_row(own, own) < (top_k + 3) / 4 ? own : INFINITY);
    }
    if (all < kMaxTop) top[all] = 0;
    if constexpr (W > 1) {
      const float v8 = wave_reduce<OpMax, 1, 8>(own);
      if (lane % 8 == 0) red[threadIdx.x / 8] = v8;
    }
    __syncthreads();
    if constexpr (W > 1) {
      const float v0 = red[2 * (lane % 16)], v1 = red[2 * (lane % 16) + 1], v = OpMax::of(v0, v1);
      m = wave_reduce<OpMax, 1, 16>(v);
      if (KT > 8 && top_k > 8) cut = kth_of_32(v0, v1, top_k);
      else if (KT > 0) cut = wave_reduce<OpMin, 1, 16>(above_in_row(v, v) < top_k ? v : INFINITY);
    }
    int count = 0;  // keys listed by this wavefront's part of the team
    cut = fmaxf(cut, -3.402823466e38f);  // -inf stays out
    if (KT > 0 && top_k > 0) {
#pragma unroll
      for (int g = 0; g < C::G; ++g) {
        if (!x.has(g) || __ballot(piece[g] >= cut) == 0) continue;
#pragma unroll
        for (int i = 0; i < C::V; ++i) {
          const float v = x.at(g, i);
          const bool in = v >= cut;
          uint64_t mask = __ballot(in);
          if (mask == 0) continue;
          if constexpr (L < 64) mask = mask >> (team * L) & ((1ull << L) - 1);
          if (in) {
            const int before = L < 64 ? __popc((uint32_t)mask & ((1u << lane) - 1))
                                      : (int)__builtin_amdgcn_mbcnt_hi(
                                            (uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
            const int at = count + before;
            if (at < kList) list[at] = rank_key(v, (uint32_t)(k0 + x.place(g) + i));
          }
          count += __popcll(mask);
        }
      }
    }
    // the sums: the largest are counted and left out (only pieces that hold
    // one are searched)
    ExpSums sum(m);
    float eq = 0.f;
#pragma unroll
    for (int g = 0; g < C::G; ++g) {
      if (!x.has(g)) continue;
      if (__ballot(piece[g] == m) != 0) {
#pragma unroll
        for (int i = 0; i < C::V; ++i) {
          const bool largest = x.at(g, i) == m;
          eq += largest ? 1.f : 0.f;
          sum.add(largest ? -INFINITY : x.at(g, i));
        }
      } else {
#pragma unroll
        for (int i = 0; i < C::V; ++i) sum.add(x.at(g, i));
      }
    }
    float s = sum.s, a = sum.a;
    s = wave_reduce<OpAdd, 1, L>(s);
    a = wave_reduce<OpAdd, 1, L>(a) * 0.69314718055994530942f;
    if (__ballot(eq != 0.f) != 0) eq = wave_reduce<OpAdd, 1, L>(eq);  // at most 8192: exact
    if constexpr (W > 1) {
      if (lane == 0) {
        sums[0][wave] = s;
        sums[1][wave] = a;
        sums[2][wave] = eq;
        counts[wave] = count;
      }
    }
    __syncthreads();
    if (KT > 0 && top_k > 0) {
      int largest = count;
      if constexpr (W > 1) largest = max(max(counts[0], counts[1]), max(counts[2], counts[3]));
      if (m != m || largest > kRanked) {
        const bool listed = m == m && largest <= kList;
        uint64_t last = ~0ull;
        for (int j = 0; j < top_k; ++j) {
          uint64_t best = 0;
          if (listed) {
#pragma nounroll
            for (int i = lane; i < count; i += L) {
              const uint64_t key = list[i];
              if (key < last && key > best) best = key;
            }
          } else {
#pragma nounroll
            for (uint32_t k = k0 + all; k < (uint32_t)(k0 + x.len); k += L * W) {  // (past the row it may pass 2^31)
              const float v = ld(row + k);
              const uint64_t key = rank_key(v, k);
              if (!(v == -INFINITY) && key < last && key > best) best = key;
            }
          }
          best = wave_max_key<L>(best);
          if constexpr (W > 1) {
            if (lane == 0) most[j & 1][wave] = best;
            __syncthreads();
            best = max(max(most[j & 1][0], most[j & 1][1]), max(most[j & 1][2], most[j & 1][3]));
          }
          last = best;
          if (all == 0) top[j] = best;
        }
      } else {
        for (int i = lane; i < count; i += L) {
          const uint64_t own_key = list[i];
          int above = 0;
          for (int w = 0; w < W; ++w) {
            const uint64_t* other = W == 1 ? list : lists[w];
            const int have = W == 1 ? count : counts[w];
            for (int j = 0; j < have; ++j) above += other[j] > own_key;
          }
          if (above < top_k) top[above] = own_key;
        }
      }
      __syncthreads();
    }
    if (wave == 0 && live) {
      if constexpr (W > 1) {
        s = (sums[0][0] + sums[0][1]) + (sums[0][2] + sums[0][3]);
        a = (sums[1][0] + sums[1][1]) + (sums[1][2] + sums[1][3]);
        eq = (sums[2][0] + sums[2][1]) + (sums[2][2] + sums[2][3]);
      }
      const Part p{m, m == -INFINITY ? 0.f : s + (eq - 1.f), a};
      if (parts == 1) {
        write_row(lane, r, lab, top_k, p, top, o);
      } else {
        const int64_t item = r * parts + blockIdx.x;
        if (lane == 0) part_out[item] = make_float4(p.m, p.t, p.a, 0.f);
        if (lane < top_k) keys_out[item * top_k + lane] = top[lane];
      }
    }
    __syncthreads();  // the next turn writes the LDS again
  }
}

// Joins the parts of a row, one wavefront per row; lane l has the parts l, l +
// 64, .. .  The best classes of up to 64 parts: keys below the top_k-th best of
// the lists' heads (as in k_scores_chunk) are out, the others are ranked.  Of
// more parts, or where more than kRanked keys are left, they come off the heads
// one by one: of 64 lists, or of 63 more and of the list so far (lane 63).
// Latency: 7 us for 64 parts with 16 best classes (one by one: 10).
template <typename T>
__global__ __launch_bounds__(64) void k_scores_join(const T* __restrict__ z, int64_t ldz, int64_t n, int classes,
                                                    int parts, const int32_t* __restrict__ labels, int top_k,
                                                    Outputs o, const float4* __restrict__ part_in,
                                                    const uint64_t* __restrict__ keys_in) {
  constexpr int kRanked = 128;
  __shared__ uint64_t list[64 * kMaxTop], left[kRanked], top[kMaxTop];
  const int lane = threadIdx.x;
  for (int64_t r = blockIdx.x; r < n; r += gridDim.x) {
    // what the row needs from memory, all of it before the first wait
    const int first = min(parts, 64) * top_k;  // keys of the first 64 parts
    uint64_t key[kMaxTop];
#pragma unroll
    for (int i = 0; i < kMaxTop; ++i) {
      if (i * 64 >= first) break;
      key[i] = lane + i * 64 < first ? keys_in[r * parts * top_k + lane + i * 64] : 0;
    }
    const Label lab = label_of(z + r * ldz, labels, r, classes);
    Part p{-INFINITY, 0.f, 0.f};
    for (int c = lane; c < parts; c += 64) {
      const float4 q = part_in[r * parts + c];
      p = c < 64 ? Part{q.x, q.y, q.z} : join(p, Part{q.x, q.y, q.z});
    }
    // the lanes' parts: values below the maximum shift by d, and of several
    // parts that hold it one goes without it
    const float m = wave_reduce<OpMax>(p.m), d = p.m - m;
    const bool holds = p.m == m, some = p.m > -INFINITY;
    const float e = expf(d), all = 1.f + p.t;
    const float t = wave_reduce<OpAdd>(holds ? p.t : some ? e * all : 0.f);
    const float a = wave_reduce<OpAdd>(holds ? p.a : some ? e * (p.a + fmaxf(d, -200.f) * all) : 0.f);
    const Part row{m, m == -INFINITY ? 0.f : t + (float)(__popcll(__ballot(holds)) - 1), m == -INFINITY ? 0.f : a};
    if (lane < kMaxTop) top[lane] = 0;
#pragma unroll
    for (int i = 0; i < kMaxTop; ++i) {
      if (i * 64 >= first) break;
      list[lane + i * 64] = key[i];
    }
    __syncthreads();
    if (top_k > 0) {
      int count = 0;
      if (parts <= 64) {
        const uint32_t head = lane < parts ? (uint32_t)(list[lane * top_k] >> 32) : 0;
        const float v = head == 0 ? -INFINITY : head == 0xfffffffeu ? INFINITY : key_value((uint64_t)head << 32);
        const float cut = wave_reduce<OpMin>(above_in_row(v, v) < (top_k + 3) / 4 ? v : INFINITY);
        const uint32_t least = (uint32_t)(rank_key(cut, 0) >> 32);
#pragma unroll
        for (int i = 0; i < kMaxTop; ++i) {
          if (i * 64 >= first) break;
          const bool in = key[i] != 0 && (uint32_t)(key[i] >> 32) >= least;
          const uint64_t mask = __ballot(in);
          if (in) {
            const int at = count + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32),
                                                                  __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
            if (at < kRanked) left[at] = key[i];
          }
          count += __popcll(mask);
        }
        __syncthreads();
      }
      if (parts <= 64 && count <= kRanked) {
        for (int i = lane; i < count; i += 64) {
          const uint64_t own = left[i];
          int above = 0;
          for (int j = 0; j < count; ++j) above += left[j] > own;
          if (above < top_k) top[above] = own;
        }
        __syncthreads();
      } else {
        for (int c0 = 0; c0 < parts;) {
          const int lists = min(parts - c0, c0 == 0 ? 64 : 63), carry = c0 == 0 ? 0 : 1;
          if (carry) {
            const uint64_t* from = keys_in + (r * parts + c0) * top_k;
            for (int i = lane; i < lists * top_k; i += 64) list[i] = from[i];
            if (lane < top_k) list[63 * kMaxTop + lane] = top[lane];
            __syncthreads();
          }
          const uint64_t* mine = lane < lists ? list + lane * top_k : list + 63 * kMaxTop;
          const bool have = lane < lists || (carry && lane == 63);
          uint64_t head = have ? mine[0] : 0;
          int at = 0;  // entries taken off this lane's list
          for (int j = 0; j < top_k; ++j) {
            const uint64_t win = wave_max_key(head);
            if (lane == 0) top[j] = win;
            if (win != 0 && head == win) head = ++at < top_k ? mine[at] : 0;
          }
          __syncthreads();
          c0 += lists;
        }
      }
    }
    write_row(lane, r, lab, top_k, row, top, o);
    __syncthreads();
  }
}

// ------------------------------------------------------------- short rows
// One thread per row of at most NC classes, the row in its registers.  A
// wavefront reads 64 consecutive rows with 16-byte loads at each row's own
// alignment (the hardware takes any), a row's loads back to back so that the
// lines its lanes share are still in the L1.  The KT best are kept sorted by
// insertion: bf16 as keys that hold the class too, one operation a place (a
// value, class pair takes four); fp32 by strict comparisons from the lowest
// class up, so that ties stay in order.  The first is left out of t.
// 1,964,906 x 20 bf16, best 3: 39 us for 165 MB (30 at the copy rate); about 500
// vector operations a row keep the SIMDs busy for some 30 of them.  (A wavefront
// per row: 1380.)

// A row of more than NP and at most NC classes as fp32, -inf past its end, in
// pieces of 16 bytes.  A cut last piece runs into what follows the row (and is
// cut off below); where that is the end of the matrix, `last`, pieces are moved
// back into it, and those few rows read again value by value.  There is no
// branch between the loads: around one the compiler waits for it before the
// next goes out.
template <typename T, int NP, int NC>
__device__ __forceinline__ void load_row(const T* __restrict__ row, const T* __restrict__ last, bool one_piece,
                                         int classes, float (&x)[NC]) {
  constexpr int V = 16 / (int)sizeof(T);
  uint32_t w[NC / V][4];
  const int room = (int)min<int64_t>(last - row, NC) - V;  // start of the last piece that fits
  if (one_piece) {                                         // the matrix holds one: the same for every row
#pragma unroll
    for (int p = 0; p < NC / V; ++p) __builtin_memcpy(w[p], row + min(p * V, room), 16);
  }
  if (!one_piece || room < (classes - 1) / V * V) {
#pragma unroll
    for (int p = 0; p < NC / V; ++p) {
      T one[V];
#pragma unroll
      for (int i = 0; i < V; ++i) one[i] = row[min(p * V + i, classes - 1)];
      __builtin_memcpy(w[p], one, 16);
      asm volatile("" ::: "memory");  // one piece's addresses at a time: all of them took up to 70 registers
    }
  }
#pragma unroll
  for (int k = 0; k < NC; ++k) {
    const uint32_t word = sizeof(T) == 4 ? w[k / V][k % V] : w[k / V][k % V / 2];
    x[k] = __uint_as_float(sizeof(T) == 4 ? word : k % 2 ? word & 0xffff0000u : word << 16);
    if (k > NP) x[k] = k < classes ? x[k] : -INFINITY;
  }
}

// f(0), f(4), .. below NC and the number of classes, unrolled for certain (the
// row's registers have no other index): f gets the group's first class.
template <int NP, int NC, int K0 = 0, class F>
__device__ __forceinline__ void groups_of_4(int classes, const F& f) {
  if constexpr (K0 < NC) {
    if (K0 <= NP || K0 < classes) f(std::integral_constant<int, K0>{});
    groups_of_4<NP, NC, K0 + 4>(classes, f);
  }
}

// The middle of three: where in goes among a >= b, or b, or a shifted down.
__device__ __forceinline__ int32_t middle(int32_t in, int32_t a, int32_t b) {
  int32_t r;
  asm("v_med3_i32 %0, %1, %2, %3" : "=v"(r) : "v"(in), "v"(a), "v"(b));
  return r;
}

template <typename T, int NP, int NC, int KT>
__global__ __launch_bounds__(64) void k_scores_rows(const T* __restrict__ z, int64_t ldz, int64_t n, int classes,
                                                    const int32_t* __restrict__ labels, int top_k, uint32_t magic,
                                                    Outputs o) {
  // the best classes of the 64 rows are 64 top_k consecutive values: they go
  // out through LDS, each lane's an odd number of words apart
  constexpr int kStride = KT | 1;
  __shared__ uint32_t stage[KT > 1 ? 2 : 1][KT > 1 ? 64 * kStride : 1];
  const int64_t r0 = (int64_t)blockIdx.x * 64;
  const int rows = (int)min<int64_t>(64, n - r0);
  const int64_t r = r0 + min((int)threadIdx.x, rows - 1);  // a last lane without a row repeats the last one
  const bool live = (int)threadIdx.x < rows;
  const T* row = z + r * ldz;
  float x[NC];
  load_row<T, NP, NC>(row, z + (n - 1) * ldz + classes, (n - 1) * ldz + classes >= 16 / (int)sizeof(T), classes, x);
  const Label label = label_of(row, labels, r, classes);
  const int lab = label.k;
  const float xl = label.x;
  float m = -INFINITY;  // NaN if the row holds one
  float tv[KT];
  int ti[KT];
  if constexpr (sizeof(T) == 2) {
    // value and class as one whole number: the value's 16 bits so that they
    // order as a signed number, below them the class, the lowest largest
    int32_t key[KT];
#pragma unroll
    for (int j = 0; j < KT; ++j) key[j] = INT32_MIN;
    groups_of_4<NP, NC>(classes, [&](auto k0) {
#pragma unroll
      for (int k = k0; k < k0 + 4; ++k) {
        m = OpMax::of(m, x[k]);
        const int32_t bits = (int32_t)__float_as_uint(x[k] + 0.f);  // -0 is 0
        const int32_t in = (bits ^ ((bits >> 31) & 0x7fff0000)) + (NC - 1 - k);
#pragma unroll
        for (int j = KT - 1; j > 0; --j) key[j] = middle(in, key[j - 1], key[j]);
        key[0] = max(key[0], in);
      }
    });
#pragma unroll
    for (int j = 0; j < KT; ++j) {
      const int32_t top = key[j] & (int32_t)0xffff0000;
      tv[j] = __uint_as_float((uint32_t)(top ^ ((top >> 31) & 0x7fff0000)));
      ti[j] = NC - 1 - (key[j] & 0xffff);
    }
  } else {
#pragma unroll
    for (int j = 0; j < KT; ++j) {
      tv[j] = -INFINITY;
      ti[j] = -1;
    }
    groups_of_4<NP, NC>(classes, [&](auto k0) {
#pragma unroll
      for (int k = k0; k < k0 + 4; ++k) {
        const float v = x[k];  // -inf past the end: above nothing
        m = OpMax::of(m, v);
        bool above[KT];
#pragma unroll
        for (int j = 0; j < KT; ++j) above[j] = v > tv[j];
#pragma unroll
        for (int j = KT - 1; j > 0; --j) {
          ti[j] = above[j - 1] ? ti[j - 1] : above[j] ? k : ti[j];
          tv[j] = __builtin_amdgcn_fmed3f(v, tv[j - 1], tv[j]);
        }
        ti[0] = above[0] ? k : ti[0];
        tv[0] = fmaxf(tv[0], v);
      }
    });
  }
  ExpSums sum(m);
  const float base = sum.base;
  groups_of_4<NP, NC>(classes, [&](auto k0) {
#pragma unroll
    for (int k = k0; k < k0 + 4; ++k) sum.add(k == ti[0] ? -INFINITY : x[k]);
  });
  const Part p{m, sum.s, sum.a * 0.69314718055994530942f};
  const float2 lh = finish(p);
  if (live) {
    if (o.logprob) o.logprob[r] = lab < 0 ? 0.f : (xl - base) - lh.x;
    o.entropy[r] = lh.y;
    reinterpret_cast<float2*>(o.stats)[r] = make_float2(m, lh.x);
  }
  if (top_k == 0) return;
  if (m != m) {  // a NaN, which the comparisons passed over: one more pass per class
    uint64_t last = ~0ull;
#pragma unroll
    for (int j = 0; j < KT; ++j)
      if (j < top_k) {
        uint64_t best = 0;
#pragma nounroll
        for (int k = 0; k < classes; ++k) {
          const uint64_t key = rank_key(ld(row + k), (uint32_t)k);
          if (key < last && key > best) best = key;
        }
        last = best;
        ti[j] = (int32_t)key_class(best);
        tv[j] = NAN;
      }
  } else if (sizeof(T) == 4) {
    int fill = 0;  // fewer classes above -inf than asked for: the lowest of the others follow
#pragma unroll
    for (int j = 0; j < KT; ++j)
      if (j < top_k && tv[j] == -INFINITY) {
        for (bool listed = true; listed;) {
          listed = false;
#pragma unroll
          for (int i = 0; i < KT; ++i) listed |= tv[i] > -INFINITY && ti[i] == fill;
          fill += listed;
        }
        ti[j] = fill++;
      }
  }
  if constexpr (KT == 1) {
    if (live) {
      o.top_index[r] = ti[0];
      o.top_logprob[r] = (tv[0] - base) - lh.x;
    }
  } else {
#pragma unroll
    for (int j = 0; j < KT; ++j)
      if (j < top_k) {
        stage[0][threadIdx.x * kStride + j] = (uint32_t)ti[j];
        stage[1][threadIdx.x * kStride + j] = __float_as_uint((tv[j] - base) - lh.x);
      }
    __syncthreads();
    for (int i = threadIdx.x; i < rows * top_k; i += 64) {
      const int at = (int)(((uint32_t)i * magic) >> 20);  // i / top_k, exact for i < 1024
      const int from = at * kStride + (i - at * top_k);
      o.top_index[r0 * top_k + i] = (int32_t)stage[0][from];
      o.top_logprob[r0 * top_k + i] = __uint_as_float(stage[1][from]);
    }
  }
}

// Which kernel takes rows of more than kRowMax classes, by their length (and,
// for rows of several chunks, by how many rows there are): the fewest lanes
// that hold the row at 32 values each, or 64 within a wavefront, since what a
// team does once per row (its reductions, the best classes' ranks) is as much
// work for 64 values as for 2048.  (40,000 rows of 512 and 513 bf16, best 8: 25
// and 44 us; 20,000 of 4096 and 4097: 61 and 72; 20,000 of 2049 fp32 by a
// wavefront each 45, by four 73.)
struct Route {
  int lanes, per_lane;  // L W, E
  int parts;            // chunks of a row
};
Route route_of(int64_t n, int classes) {
  if (classes <= 512) return {16, 32, 1};
  if (classes <= 2048) return {64, 32, 1};
  if (classes <= 4096) return {64, 64, 1};
  if (classes <= 8192) return {256, 32, 1};
  // chunks of 8192 once they are enough workgroups for 256 CUs, else four times
  // as many (102 and 103 rows of 40001 bf16, best 8, one rule each: 14 and 13 us)
  const int big = (int)ceil_div(classes, 8192);
  return n * big >= 512 ? Route{256, 32, big} : Route{256, 8, (int)ceil_div(classes, 2048)};
}

// Whether one thread takes a row: of up to 64 classes; up to 128 in bf16, whose
// best classes cost a thread less, and in fp32 where there is a wavefront of rows
// for every SIMD.  By threads and by teams of 16 lanes, us (17 is the host's time
// of a call, and what shorter kernels show):
//   fp32                32,768 x 70  x 128    65,536 x 70  x 128    262,144 x 70   x 128
//     best 3               17, 17    17, 17      17, 17    17, 18       23, 53     38, 62
//     best 8               17, 17    19, 17      17, 20    21, 21       32, 62     51, 70
//     best 16              17, 17    28, 19      21, 30    34, 31       50, 104    84, 113
//   bf16, best 8           17, 18    17, 17      17, 30    17, 22       24, 97     31, 68
//     best 16              17, 30    17, 20      17, 51    17, 36       28, 186    38, 126
// (16,384 rows: 17 but for best 16: fp32 x 128 by threads 25, bf16 x 70 by teams 22.)
constexpr int kRowMax = 64;
template <typename T>
bool by_thread(int64_t n, int classes) {
  return classes <= kRowMax || (classes <= 128 && (sizeof(T) == 2 || n >= 1 << 16));
}

// f(NP, NC) for rows of more than NP and at most NC classes.
template <class F>
void by_classes(int classes, const F& f) {
  if (classes <= 16) f(std::integral_constant<int, 0>{}, std::integral_constant<int, 16>{});
  else if (classes <= 24) f(std::integral_constant<int, 16>{}, std::integral_constant<int, 24>{});
  else if (classes <= 32) f(std::integral_constant<int, 24>{}, std::integral_constant<int, 32>{});
  else if (classes <= 48) f(std::integral_constant<int, 32>{}, std::integral_constant<int, 48>{});
  else if (classes <= 64) f(std::integral_constant<int, 48>{}, std::integral_constant<int, 64>{});
  else f(std::integral_constant<int, 64>{}, std::integral_constant<int, 128>{});
}

template <typename T, int NP, int NC>
void launch_rows(const T* z, int64_t ldz, int64_t n, int classes, const int32_t* labels, int top_k, const Outputs& o,
                 hipStream_t s) {
  const unsigned g = (unsigned)ceil_div(n, 64);
  const uint32_t magic = top_k > 0 ? ((1u << 20) + top_k - 1) / top_k : 0;
  if (top_k <= 1)
    k_scores_rows<T, NP, NC, 1><<<g, 64, 0, s>>>(z, ldz, n, classes, labels, top_k, magic, o);
  else if (top_k <= 3)
    k_scores_rows<T, NP, NC, 3><<<g, 64, 0, s>>>(z, ldz, n, classes, labels, top_k, magic, o);
  else if (top_k <= 8)
    k_scores_rows<T, NP, NC, 8><<<g, 64, 0, s>>>(z, ldz, n, classes, labels, top_k, magic, o);
  else
    k_scores_rows<T, NP, NC, 16><<<g, 64, 0, s>>>(z, ldz, n, classes, labels, top_k, magic, o);
}

template <typename T>
sscn_status launch_scores(const T* z, int64_t ldz, int64_t n, int classes, const int32_t* labels, int top_k,
                          const Outputs& o, void* workspace, hipStream_t s) {
  if (by_thread<T>(n, classes)) {
    by_classes(classes, [&](auto np, auto nc) {
      launch_rows<T, decltype(np)::value, decltype(nc)::value>(z, ldz, n, classes, labels, top_k, o, s);
    });
    SSCN_HIP(hipGetLastError());
    return SSCN_OK;
  }
  const Route w = route_of(n, classes);
  const int64_t items = n * w.parts;
  float4* parts = (float4*)workspace;
  uint64_t* keys = (uint64_t*)(parts + items);
  // a workgroup takes rows in turn once there are some 16384 of them
  const unsigned by_team = (unsigned)std::min<int64_t>(ceil_div(n, 64 / std::min(w.lanes, 64)), 16384);
  const dim3 by_part((unsigned)w.parts, (unsigned)std::max<int64_t>(1, std::min<int64_t>(n, 16384 / w.parts)));
  const auto run = [&](auto kt) {
    constexpr int KT = decltype(kt)::value;
    if (w.lanes == 16)
      k_scores_chunk<T, 16, 1, 32, KT><<<by_team, 64, 0, s>>>(z, ldz, n, classes, labels, top_k, o, parts, keys);
    else if (w.lanes == 64 && w.per_lane == 64)
      k_scores_chunk<T, 64, 1, 64, KT><<<by_team, 64, 0, s>>>(z, ldz, n, classes, labels, top_k, o, parts, keys);
    else if (w.lanes == 64)
      k_scores_chunk<T, 64, 1, 32, KT><<<by_team, 64, 0, s>>>(z, ldz, n, classes, labels, top_k, o, parts, keys);
    else if (w.per_lane == 32)
      k_scores_chunk<T, 64, 4, 32, KT><<<by_part, 256, 0, s>>>(z, ldz, n, classes, labels, top_k, o, parts, keys);
    else
      k_scores_chunk<T, 64, 4, 8, KT><<<by_part, 256, 0, s>>>(z, ldz, n, classes, labels, top_k, o, parts, keys);
  };
  if (top_k == 0)
    run(std::integral_constant<int, 0>{});
  else if (top_k <= 8)
    run(std::integral_constant<int, 8>{});
  else
    run(std::integral_constant<int, 16>{});
  SSCN_HIP(hipGetLastError());
  if (w.parts > 1) {
    k_scores_join<T><<<(unsigned)std::min<int64_t>(n, 16384), 64, 0, s>>>(z, ldz, n, classes, w.parts, labels, top_k, o,
                                                                          parts, keys);
    SSCN_HIP(hipGetLastError());
  }
  return SSCN_OK;
}

// ------------------------------------------------------------- the gradient
// With A_k what class k receives directly (g = dlogprob where k is the label,
// dtop_j where k is the j-th best class), G their sum and h = dentropy,
//   dx_k = -A_k expm1(log p_k) - p_k ((G - A_k) + h (log p_k + H)),
// which is A_k - p_k (G + h (log p_k + H)) without that form's cancellation
// where p_k is close to 1.  All but the label and the best classes have A_k = 0:
// they are written as -p_k (G + h (log p_k + H)), and then those few again.
struct GradInputs {
  const int32_t* labels;
  const float *stats, *entropy;
  int top_k;                // 0 unless dtop is given
  const int32_t* top_index;
  const float *dlogprob, *dentropy, *dtop;
};
struct GradRow {
  float base, L, h, H, g, G;
  int lab;
  bool empty;
};
// direct: the sum of the row's dtop.
__device__ __forceinline__ GradRow grad_row(const GradInputs& q, int64_t r, int classes, float direct) {
  GradRow w;
  const float2 st = reinterpret_cast<const float2*>(q.stats)[r];
  w.L = st.y;
  w.empty = st.x == -INFINITY && st.y == 0.f;
  w.base = w.empty ? 0.f : st.x;
  w.h = q.dentropy ? q.dentropy[r] : 0.f;
  w.H = q.dentropy ? q.entropy[r] : 0.f;
  w.lab = q.dlogprob ? q.labels[r] : -1;
  w.g = w.lab < 0 ? 0.f : w.lab >= classes ? NAN : q.dlogprob[r];
  w.G = w.g + direct;
  if (w.L != w.L) w.G = NAN;  // the clamp below would lose it
  if (w.empty) {
    w.g = w.h = 0.f;
    w.G = w.lab >= classes ? NAN : 0.f;  // the row's gradient, NaN where its log probability is
  }
  return w;
}
__device__ __forceinline__ float grad_dense(const GradRow& w, float x) {
  const float lp = fmaxf((x - w.base) - w.L, -300.f);  // e^-300 is 0: no 0 * inf
  return -__builtin_amdgcn_exp2f(lp * 1.44269504088896340736f) * fmaf(w.h, lp + w.H, w.G);
}
__device__ __forceinline__ float grad_direct(const GradRow& w, float x, float A) {
  if (w.empty) return w.G;
  const float lp = (x - w.base) - w.L, p = expf(lp);
  return -A * expm1f(lp) - p * ((w.G - A) + (p == 0.f ? 0.f : w.h * (lp + w.H)));
}
// Short rows, a thread per row as in k_scores_rows.  The 64 rows of a
// wavefront go out through LDS, rows an odd number of words apart (each lane
// its own bank), as consecutive words of 4 bytes (WORDS) or single values.
// KT: at least top_k; the rows' best classes and their gradients come in
// through LDS the same way.  1,964,906 x 20 bf16: 43 us for 204 MB, 4.7 TB/s,
// memory-bound (a wavefront per row: 520); with 4 best classes' gradients 72.
template <typename T, int NP, int NC, bool WORDS, int KT>
__global__ __launch_bounds__(64) void k_grad_rows(const T* __restrict__ z, int64_t ldz, int64_t n, int classes,
                                                  GradInputs q, T* __restrict__ dz, int64_t ldd, int stride,
                                                  uint32_t magic, uint32_t top_magic) {
  extern __shared__ uint32_t lds[];
  constexpr int kStride = KT | 1;
  __shared__ uint32_t stage[KT ? 2 : 1][KT ? 64 * kStride : 1];
  const int64_t r0 = (int64_t)blockIdx.x * 64;
  const int rows = (int)min<int64_t>(64, n - r0);
  const int64_t r = r0 + min((int)threadIdx.x, rows - 1);  // a last lane without a row repeats the last one
  T* out = reinterpret_cast<T*>(lds + threadIdx.x * stride);
  const T* row = z + r * ldz;
  float x[NC];
  load_row<T, NP, NC>(row, z + (n - 1) * ldz + classes, (n - 1) * ldz + classes >= 16 / (int)sizeof(T), classes, x);
  int ti[KT ? KT : 1];
  float tv[KT ? KT : 1], direct = 0.f;
  if constexpr (KT > 0) {
    for (int i = threadIdx.x; i < rows * q.top_k; i += 64) {
      const int at = (int)(((uint32_t)i * top_magic) >> 20);  // i / top_k, exact for i < 1024
      const int to = at * kStride + (i - at * q.top_k);
      stage[0][to] = (uint32_t)q.top_index[r0 * q.top_k + i];
      stage[1][to] = __float_as_uint(q.dtop[r0 * q.top_k + i]);
    }
    __syncthreads();
    const int mine = min((int)threadIdx.x, rows - 1) * kStride;
#pragma unroll
    for (int j = 0; j < KT; ++j) {
      ti[j] = j < q.top_k ? (int)stage[0][mine + j] : -1;
      tv[j] = j < q.top_k ? __uint_as_float(stage[1][mine + j]) : 0.f;
      direct += tv[j];
    }
  }
  const GradRow w = grad_row(q, r, classes, direct);
  groups_of_4<NP, NC>(classes, [&](auto k0) {
#pragma unroll
    for (int k = k0; k < k0 + 4; ++k) x[k] = grad_dense(w, x[k]);
    // whole words: the stride has room for a last group's unused values
    if constexpr (sizeof(T) == 4) {
      __builtin_memcpy(out + k0, x + k0, 16);
    } else {
      const uint32_t v[2] = {pack_bf16(x[k0], x[k0 + 1]), pack_bf16(x[k0 + 2], x[k0 + 3])};
      __builtin_memcpy(out + k0, v, 8);
    }
  });
  if (w.lab >= 0 && w.lab < classes) {
    float A = w.g;
#pragma unroll
    for (int j = 0; j < KT; ++j) A += ti[j] == w.lab ? tv[j] : 0.f;
    st(out + w.lab, grad_direct(w, ld(row + w.lab), A));
  }
  if constexpr (KT > 0) {
#pragma unroll
    for (int i = 0; i < KT; ++i)
      if (ti[i] >= 0 && ti[i] < classes) {
        float A = ti[i] == w.lab ? w.g : 0.f;
#pragma unroll
        for (int j = 0; j < KT; ++j) A += ti[j] == ti[i] ? tv[j] : 0.f;
        st(out + ti[i], grad_direct(w, ld(row + ti[i]), A));
      }
  }
  __syncthreads();
  const int per = WORDS ? classes * (int)sizeof(T) / 4 : classes;  // items of a row
  for (int i = threadIdx.x; i < rows * per; i += 64) {
    const int at_row = (int)(((uint32_t)i * magic) >> 20), at = i - at_row * per;  // i / per, exact for i < 4096
    T* to = dz + (r0 + at_row) * ldd;
    if constexpr (WORDS)
      reinterpret_cast<uint32_t*>(to)[at] = lds[at_row * stride + at];
    else
      to[at] = reinterpret_cast<const T*>(lds + at_row * stride)[at];
  }
}

// Longer rows, teams as in k_scores_chunk, `span` values of a row to a team;
// nothing is kept, so a team walks its span piece by piece.  Every 16 lanes
// hold the row's best classes and their gradients, one a lane.  1024 x 40001
// fp32: 65 us for 328 MB, 5.0 TB/s, memory-bound.
template <typename T, int L, int W>
__global__ __launch_bounds__(64 * W) void k_grad_chunk(const T* __restrict__ z, int64_t ldz, int64_t n, int classes,
                                                       int span, GradInputs q, T* __restrict__ dz, int64_t ldd) {
  constexpr int V = 16 / (int)sizeof(T), kTeams = 64 / L;
  const int team = (threadIdx.x & 63) / L, all = W == 1 ? threadIdx.x & (L - 1) : (int)threadIdx.x;
  const int64_t rows = W == 1 ? (int64_t)gridDim.x * kTeams : gridDim.y;
  const int k0 = W == 1 ? 0 : (int)blockIdx.x * span, len = min(classes - k0, span);
  for (int64_t r0 = W == 1 ? (int64_t)blockIdx.x * kTeams : blockIdx.y; r0 < n; r0 += rows) {
    const int64_t r = r0 + team;
    const T* row = z + r * ldz;
    T* to = dz + r * ldd;
    constexpr int G = 2, kStep = L * W * V;  // pieces in flight
    uint32_t b[G][4];
    const int first = all * V;
    const auto load = [&](int kb) {
#pragma unroll
      for (int g = 0; g < G; ++g)  // a cut piece is the V values up to the span's end
        __builtin_memcpy(b[g], row + k0 + min(kb + g * kStep, len - V), 16);
    };
    if (r < n) load(first);  // before what the row's numbers wait for
    GradRow w{};
    const int j = threadIdx.x & 15;
    const bool has = r < n && j < q.top_k;
    const int cls = has ? q.top_index[r * q.top_k + j] : -1;
    const float t = has ? q.dtop[r * q.top_k + j] : 0.f;
    if (r < n) {
      w = grad_row(q, r, classes, wave_reduce<OpAdd, 1, 16>(t));
      for (int kb = first; kb < len;) {
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const int k = kb + g * kStep, at = k0 + min(k, len - V);
          if (k >= len) break;
          float v[V];
#pragma unroll
          for (int i = 0; i < V; ++i)
            v[i] = grad_dense(w, sizeof(T) == 4 ? __uint_as_float(b[g][i % 4])
                                 : i % 2        ? __uint_as_float(b[g][i / 2] & 0xffff0000u)
                                                : __uint_as_float(b[g][i / 2] << 16));
#pragma unroll
          for (int i = 0; i < 4; ++i)
            b[g][i] = sizeof(T) == 4 ? __float_as_uint(v[i]) : pack_bf16(v[2 * i % V], v[(2 * i + 1) % V]);
          if (k + V <= len) {  // one store, at whatever alignment it has
            __builtin_memcpy(to + at, b[g], 16);
          } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
              if (at + i >= k0 + k) st(to + at + i, v[i]);
          }
        }
        kb += G * kStep;
        if (kb < len) load(kb);
      }
    }
    __syncthreads();  // the team's stores come before those below
    const bool mine = cls >= k0 && cls < k0 + len, label_here = r < n && w.lab >= k0 && w.lab < k0 + len;
    if (all < 16 && __ballot(mine || label_here) != 0) {
      const Same same = same_in_row(cls, t);
      const float A = t + same.sum, to_label = w.g + wave_reduce<OpAdd, 1, 16>(cls == w.lab ? t : 0.f);
      if (mine && cls != w.lab && !same.before) st(to + cls, grad_direct(w, ld(row + cls), A));
      if (label_here && all == 0) st(to + w.lab, grad_direct(w, ld(row + w.lab), to_label));
    }
  }
}

template <typename T, int NP, int NC>
void launch_grad_rows(const T* z, int64_t ldz, int64_t n, int classes, const GradInputs& q, T* dz, int64_t ldd,
                      hipStream_t s) {
  const int bytes = (int)sizeof(T) * classes;
  const bool words = bytes % 4 == 0 && ldd * sizeof(T) % 4 == 0 && reinterpret_cast<uintptr_t>(dz) % 4 == 0;
  const int stride = (int)(ceil_div(classes, 4) * 4 * sizeof(T) / 4) | 1;
  const int per = words ? bytes / 4 : classes;
  const uint32_t magic = ((1u << 20) + per - 1) / per;
  const uint32_t top_magic = q.top_k > 0 ? ((1u << 20) + q.top_k - 1) / q.top_k : 0;
  const unsigned g = (unsigned)ceil_div(n, 64);
  const size_t lds = (size_t)64 * stride * 4;
  const auto run = [&](auto words_t) {
    constexpr bool WORDS = decltype(words_t)::value;
    if (q.top_k == 0)
      k_grad_rows<T, NP, NC, WORDS, 0><<<g, 64, lds, s>>>(z, ldz, n, classes, q, dz, ldd, stride, magic, top_magic);
    else if (q.top_k <= 4)
      k_grad_rows<T, NP, NC, WORDS, 4><<<g, 64, lds, s>>>(z, ldz, n, classes, q, dz, ldd, stride, magic, top_magic);
    else
      k_grad_rows<T, NP, NC, WORDS, 16><<<g, 64, lds, s>>>(z, ldz, n, classes, q, dz, ldd, stride, magic, top_magic);
  };
  if (words) run(std::true_type{});
  else run(std::false_type{});
}

// Which kernel takes the gradient's rows, by their length: a thread, 16 lanes, a
// wavefront, a workgroup per 2048 values.  Both sides of the lines, us, without
// and with 4 best classes' gradients (fp32; bf16):
//    64 classes, 300,000 rows: by threads 44, 57; 22, 32   by 16 lanes 55, 64; 40, 52
//   512 classes,  40,000 rows: by 16 lanes 40, 46; 18, 21  by wavefronts 41, 45; 25, 30
//   513 classes,  40,000 rows: by 16 lanes 55, 60; 25, 29  by wavefronts 47, 52; 31, 35
//  2048 classes,  10,000 rows: by wavefronts 40, 43; 17, 19  (by workgroups from 1025 on: 36, 37; 22, 24)
//  2049 classes,  10,000 rows: by wavefronts 48, 50; 23, 25  by workgroups 61, 65; 43, 47
//  4096 classes,  10,000 rows: by wavefronts 78, 81; 38, 40  by workgroups 63, 67; 48, 53
// The lines are fp32's, a little early above 2048; bf16's, of half the bytes, would
// lie at some 1024 and past 4096.
template <typename T>
sscn_status launch_grad(const T* z, int64_t ldz, int64_t n, int classes, const GradInputs& q, T* dz, int64_t ldd,
                        hipStream_t s) {
  if (classes <= kRowMax) {
    by_classes(classes, [&](auto np, auto nc) {
      if constexpr (decltype(nc)::value <= kRowMax)
        launch_grad_rows<T, decltype(np)::value, decltype(nc)::value>(z, ldz, n, classes, q, dz, ldd, s);
    });
  } else if (classes <= 512) {
    k_grad_chunk<T, 16, 1><<<(unsigned)std::min<int64_t>(ceil_div(n, 4), 32768), 64, 0, s>>>(z, ldz, n, classes, 512, q,
                                                                                             dz, ldd);
  } else if (classes <= 2048) {
    k_grad_chunk<T, 64, 1><<<(unsigned)std::min<int64_t>(n, 32768), 64, 0, s>>>(z, ldz, n, classes, 2048, q, dz, ldd);
  } else {
    const int span = 2048;  // (8192, with a quarter of the workgroups: 78 us for 69 at 1024 x 40001 fp32)
    const int64_t parts = ceil_div(classes, span);
    const dim3 g((unsigned)parts, (unsigned)std::max<int64_t>(1, std::min<int64_t>(n, 32768 / parts)));
    k_grad_chunk<T, 64, 4><<<g, 256, 0, s>>>(z, ldz, n, classes, span, q, dz, ldd);
  }
  SSCN_HIP(hipGetLastError());
  return SSCN_OK;
}

sscn_status check_rows(const void* p, int64_t ld, int64_t n, int classes, sscn_dtype dtype) {
  if (dtype != SSCN_F32 && dtype != SSCN_BF16) return fail(SSCN_ERR_INVALID_ARG, "unknown dtype");
  if (n < 0 || classes < 1) return fail(SSCN_ERR_INVALID_ARG, "scores: n must be >= 0 and classes >= 1");
  if (n > 0 && !p) return fail(SSCN_ERR_INVALID_ARG, "scores: NULL logits or dlogits");
  if (ld < classes) return fail(SSCN_ERR_INVALID_ARG, "scores: row stride below the number of classes");
  if (reinterpret_cast<uintptr_t>(p) % (dtype == SSCN_F32 ? 4 : 2) != 0)
    return fail(SSCN_ERR_INVALID_ARG, "scores: logits or dlogits not aligned to their elements");
  return SSCN_OK;
}
sscn_status check_top(int32_t top_k, int32_t classes) {
  if (top_k < 0 || top_k > std::min<int32_t>(kMaxTop, classes))
    return fail(SSCN_ERR_INVALID_ARG, "scores: top_k must be in [0, min(16, classes)]");
  return SSCN_OK;
}

}  // namespace
}  // namespace sscn

using namespace sscn;

extern "C" sscn_status sscn_label_scores_workspace(int64_t n, int32_t classes, int32_t top_k, int64_t* bytes) {
  if (n < 0 || classes < 1) return fail(SSCN_ERR_INVALID_ARG, "scores: n must be >= 0 and classes >= 1");
  SSCN_TRY(check_top(top_k, classes));
  if (!bytes) return fail(SSCN_ERR_INVALID_ARG, "scores: NULL bytes");
  const Route w = route_of(n, classes);
  *bytes = w.parts > 1 ? n * w.parts * (int64_t)(sizeof(float4) + sizeof(uint64_t) * top_k) : 0;
  return SSCN_OK;
}

extern "C" sscn_status sscn_label_scores(const void* logits, int64_t ldz, int64_t n, int32_t classes,
                                         sscn_dtype dtype, const int32_t* labels, int32_t top_k, float* logprob,
                                         float* entropy, float* stats, int32_t* top_index, float* top_logprob,
                                         void* workspace, int64_t workspace_bytes, hipStream_t stream) {
  SSCN_TRY(check_rows(logits, ldz, n, classes, dtype));
  SSCN_TRY(check_top(top_k, classes));
  if ((labels == nullptr) != (logprob == nullptr) && n > 0)
    return fail(SSCN_ERR_INVALID_ARG, "scores: labels and logprob go together");
  if (n > 0 && (!entropy || !stats)) return fail(SSCN_ERR_INVALID_ARG, "scores: NULL entropy or stats");
  if (n > 0 && top_k > 0 && (!top_index || !top_logprob))
    return fail(SSCN_ERR_INVALID_ARG, "scores: NULL top_index or top_logprob");
  int64_t need = 0;
  SSCN_TRY(sscn_label_scores_workspace(n, classes, top_k, &need));
  if (workspace_bytes < need || (need > 0 && (!workspace || reinterpret_cast<uintptr_t>(workspace) % 16 != 0)))
    return fail(SSCN_ERR_INVALID_ARG, "scores: no workspace of the size that ..._workspace says, 16-byte aligned");
  if (n == 0) return SSCN_OK;
  const Outputs o{logprob, entropy, stats, top_index, top_logprob};
  return dtype == SSCN_F32
             ? launch_scores((const float*)logits, ldz, n, classes, labels, top_k, o, workspace, stream)
             : launch_scores((const uint16_t*)logits, ldz, n, classes, labels, top_k, o, workspace, stream);
}

extern "C" sscn_status sscn_label_scores_backward(const void* logits, int64_t ldz, int64_t n, int32_t classes,
                                                  sscn_dtype dtype, const int32_t* labels, const float* stats,
                                                  const float* entropy, int32_t top_k, const int32_t* top_index,
                                                  const float* dlogprob, const float* dentropy, const float* dtop,
                                                  void* dlogits, int64_t ldd, hipStream_t stream) {
  SSCN_TRY(check_rows(logits, ldz, n, classes, dtype));
  SSCN_TRY(check_rows(dlogits, ldd, n, classes, dtype));
  SSCN_TRY(check_top(top_k, classes));
  if (n == 0) return SSCN_OK;
  if (!stats) return fail(SSCN_ERR_INVALID_ARG, "scores: NULL stats");
  if (dlogprob && !labels) return fail(SSCN_ERR_INVALID_ARG, "scores: dlogprob without labels");
  if (dentropy && !entropy) return fail(SSCN_ERR_INVALID_ARG, "scores: dentropy without entropy");
  if (dtop && (top_k == 0 || !top_index)) return fail(SSCN_ERR_INVALID_ARG, "scores: dtop without top_index");
  if (rows_share(logits, ldz, classes, dlogits, ldd, classes, n, dtype == SSCN_F32 ? 4 : 2) || dlogits == logits)
    return fail(SSCN_ERR_INVALID_ARG, "scores: the gradient cannot replace the logits");
  const GradInputs q{labels, stats, entropy, dtop ? top_k : 0, top_index, dlogprob, dentropy, dtop};
  return dtype == SSCN_F32 ? launch_grad((const float*)logits, ldz, n, classes, q, (float*)dlogits, ldd, stream)
                           : launch_grad((const uint16_t*)logits, ldz, n, classes, q, (uint16_t*)dlogits, ldd, stream);
}
