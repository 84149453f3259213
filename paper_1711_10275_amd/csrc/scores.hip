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

// ------------------------------------------------------------- longer rows
// A row is read as 16-byte (W = 1: 4-byte) pieces at their own alignment, so
// that rows that start anywhere are read wide; the pieces at its ends that it
// shares with its neighbours are read value by value. A workgroup of W
// wavefronts holds a chunk of 64 W E values in registers, E a thread: one read
// of the logits, the maximum before the exponentials.
template <typename T, int W, int E>
struct Chunk {
  static constexpr int V = (W == 1 ? 4 : 16) / (int)sizeof(T);  // values per piece
  static constexpr int G = E / V;                               // pieces per thread
  static constexpr int kThreads = 64 * W;
  static constexpr int64_t kPieces = (int64_t)kThreads * G;     // per chunk
  static constexpr int WORDS = V * (int)sizeof(T) / 4 > 0 ? V * (int)sizeof(T) / 4 : 1;

  // Class of value i of piece g of this thread, for the chunk that starts at class c0.
  __device__ static int cls(int64_t c0, int g, int i) {
    return (int)(c0 + ((int64_t)g * kThreads + threadIdx.x) * V + i);
  }
  // Classes between the first whole piece's alignment and the row's start.
  __device__ static int head(const T* row) { return (int)(reinterpret_cast<uintptr_t>(row) % (V * sizeof(T)) / sizeof(T)); }

  // The chunk as it is stored (bf16 two to a word), and its value i of piece g.
  uint32_t w[G][WORDS];
  __device__ float at(int g, int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[g][i]);
    else return __uint_as_float(i % 2 ? w[g][i / 2] & 0xffff0000u : w[g][i / 2] << 16);
  }
  // -inf past the row's ends.  c0 = -head + chunk * kPieces * V.
  __device__ void load(const T* row, int classes, int64_t c0) {
    const int64_t wave0 = c0 + (int64_t)(threadIdx.x & ~63) * V;  // first class of this wavefront's first piece
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const int64_t first = wave0 + (int64_t)g * kThreads * V;    // uniform in the wavefront
      const int64_t k0 = first + (int64_t)(threadIdx.x & 63) * V;
      if (first >= 0 && first + 64 * V <= classes) {
        __builtin_memcpy(w[g], __builtin_assume_aligned(row + k0, V * sizeof(T)), V * sizeof(T));
      } else {
        const auto one = [&](int i) -> uint32_t {
          const bool in = k0 + i >= 0 && k0 + i < classes;
          if constexpr (sizeof(T) == 4) return in ? __float_as_uint(row[k0 + i]) : 0xff800000u;
          else return in ? row[k0 + i] : 0xff80u;
        };
#pragma unroll
        for (int i = 0; i < WORDS; ++i)
          w[g][i] = sizeof(T) == 4 ? one(i) : one(2 * i) | one(2 * i + 1) << 16;
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
__device__ __forceinline__ float2 finish(const Part& p) {
  if (p.m == INFINITY || p.m != p.m) return make_float2(NAN, NAN);
  if (p.m == -INFINITY) return make_float2(0.f, 0.f);
  const float l = log1pf(p.t);
  return make_float2(l, l - p.a / (1.f + p.t));
}

struct Outputs {
  float *logprob, *entropy, *stats;
  int32_t* top_index;
  float* top_logprob;
};

// Writes row r.  top: top_k keys in LDS, best first, 0 where the row has fewer
// classes above -inf: the lowest of the others follow.
template <typename T>
__device__ __forceinline__ void write_row(const T* row, int64_t r, int classes, const int32_t* labels, int top_k,
                                          const Part& p, uint64_t* top, const Outputs& o) {
  const int lane = threadIdx.x & 63;
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
    if (o.logprob) {
      const int lab = labels[r];
      o.logprob[r] = lab < 0 ? 0.f : lab >= classes ? NAN : (ld(row + lab) - base) - lh.x;
    }
    o.entropy[r] = lh.y;
    o.stats[2 * r] = p.m;
    o.stats[2 * r + 1] = lh.x;
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (lane < top_k) {
    const uint32_t k = key_class(top[lane]);
    o.top_index[r * top_k + lane] = (int32_t)k;
    o.top_logprob[r * top_k + lane] = (ld(row + k) - base) - lh.x;
  }
}

// One chunk of one row per turn of a workgroup; `parts` chunks per row.  With
// one the row is written, with more its Part and its best keys are left for
// k_scores_join.
//
// The best classes: T, the least of at least top_k groups' maxima (groups of
// threads that share no value), is no larger than the top_k-th best value, so
// what is below T is out.  Few values are left (about top_k log(top_k) of
// unordered ones); each counts the keys above its own, which is its rank.
// Values of -inf stay out of the list.  Masks that leave some group nothing
// make T -inf: the largest is taken off a long list top_k times.  A list that
// overflows (ties at T), or a NaN, takes them off the row itself.
template <typename T, int W, int E>
__global__ __launch_bounds__(64 * W) void k_scores_chunk(const T* __restrict__ z, int64_t ldz, int64_t n, int classes,
                                                         const int32_t* __restrict__ labels, int top_k, Outputs o,
                                                         float4* __restrict__ part_out,
                                                         uint64_t* __restrict__ keys_out) {
  using C = Chunk<T, W, E>;
  constexpr int kList = 64 * W * E < 2048 ? 64 * W * E : 2048, kRanked = 128;
  __shared__ uint64_t list[kList], top[kMaxTop], most[2][W];
  __shared__ float red[2][W], sums[3][W];
  __shared__ int count;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int parts = (int)gridDim.x;
  for (int64_t r = blockIdx.y; r < n; r += gridDim.y) {
    const T* row = z + r * ldz;
    const int64_t c0 = (int64_t)blockIdx.x * (C::kPieces * C::V) - C::head(row);
    C x;
    x.load(row, classes, c0);
    float own = -INFINITY;  // this thread's maximum
#pragma unroll
    for (int g = 0; g < C::G; ++g)
#pragma unroll
      for (int i = 0; i < C::V; ++i) own = OpMax::of(own, x.at(g, i));
    // maxima of groups of lanes, and the threshold from them
    const float v4 = wave_reduce<OpMax, 1, 4>(own), v8 = wave_reduce<OpMax, 4, 8>(v4);
    const float v16 = wave_reduce<OpMax, 8, 16>(v8), v32 = wave_reduce<OpMax, 16, 32>(v16);
    float m = wave_reduce<OpMax, 32, 64>(v32), cut = m;
    if constexpr (W == 1) {
      if (top_k > 1) cut = wave_reduce<OpMin>(top_k <= 2 ? v32 : top_k <= 4 ? v16 : top_k <= 8 ? v8 : v4);
    } else {
      static_assert(W == 4);
      if (top_k > 4) cut = wave_reduce<OpMin>(top_k <= 8 ? v32 : v16);
    }
    if (threadIdx.x == 0) count = 0;
    if (threadIdx.x < kMaxTop) top[threadIdx.x] = 0;
    if constexpr (W > 1) {
      if (lane == 0) {
        red[0][wave] = m;
        red[1][wave] = cut;
      }
    }
    __syncthreads();
    if constexpr (W > 1) {
      const float m0 = red[0][0], m1 = red[0][1], m2 = red[0][2], m3 = red[0][3];
      m = OpMax::of(OpMax::of(m0, m1), OpMax::of(m2, m3));
      const float least = fminf(fminf(red[1][0], red[1][1]), fminf(red[1][2], red[1][3]));
      // of four maxima the first, second, third or fourth largest
      const float mid0 = fminf(fmaxf(m0, m1), fmaxf(m2, m3)), mid1 = fmaxf(fminf(m0, m1), fminf(m2, m3));
      cut = top_k == 1 ? m : top_k == 2 ? fmaxf(mid0, mid1) : top_k == 3 ? fminf(mid0, mid1) : least;
    }
    if (top_k > 0 && m == m) {
#pragma unroll
      for (int g = 0; g < C::G; ++g)
#pragma unroll
        for (int i = 0; i < C::V; ++i)
          if (x.at(g, i) >= cut && x.at(g, i) > -INFINITY) {
            const int at = atomicAdd(&count, 1);
            if (at < kList) list[at] = rank_key(x.at(g, i), (uint32_t)C::cls(c0, g, i));
          }
    }
    // The sums, of 2^h with h = (x - m) log2(e): the largest are counted and
    // left out (only a wavefront that holds one looks for them).  h is one
    // rounded product: a term is off by up to 2.25 |x - m| half steps, which its
    // own size e^(x - m) outweighs; forming the product's low part too would
    // cost three more operations a value.
    float s = 0.f, a = 0.f, eq = 0.f;
    const float base = m == -INFINITY ? 0.f : m;
    const auto add = [&](float v) {
      const float h = fmaxf((v - base) * 1.44269504088896340736f, -300.f);  // 2^-300 is 0
      const float e = __builtin_amdgcn_exp2f(h);
      s += e;
      a = fmaf(e, h, a);
    };
    if (__ballot(own == m) != 0) {
#pragma unroll
      for (int g = 0; g < C::G; ++g)
#pragma unroll
        for (int i = 0; i < C::V; ++i) {
          const bool largest = x.at(g, i) == m;
          eq += largest ? 1.f : 0.f;
          add(largest ? -INFINITY : x.at(g, i));
        }
      eq = wave_reduce<OpAdd>(eq);  // at most 8192: exact
    } else {
#pragma unroll
      for (int g = 0; g < C::G; ++g)
#pragma unroll
        for (int i = 0; i < C::V; ++i) add(x.at(g, i));
    }
    s = wave_reduce<OpAdd>(s);
    a = wave_reduce<OpAdd>(a) * 0.69314718055994530942f;
    if constexpr (W > 1) {
      if (lane == 0) {
        sums[0][wave] = s;
        sums[1][wave] = a;
        sums[2][wave] = eq;
      }
    }
    __syncthreads();
    const int found = count;
    if (top_k > 0) {
      if (m != m || found > kRanked) {
        const bool listed = m == m && found <= kList;
        uint64_t last = ~0ull;
        for (int j = 0; j < top_k; ++j) {
          uint64_t best = 0;
          if (listed) {
#pragma nounroll
            for (int i = threadIdx.x; i < found; i += C::kThreads) {
              const uint64_t key = list[i];
              if (key < last && key > best) best = key;
            }
          } else {
            const int first = (int)max<int64_t>(c0, 0), end = (int)min<int64_t>(c0 + C::kPieces * C::V, classes);
#pragma nounroll
            for (int k = first + threadIdx.x; k < end; k += C::kThreads) {
              const float v = ld(row + k);
              const uint64_t key = rank_key(v, (uint32_t)k);
              if (!(v == -INFINITY) && key < last && key > best) best = key;
            }
          }
          best = wave_max_key(best);
          if constexpr (W > 1) {
            if (lane == 0) most[j & 1][wave] = best;
            __syncthreads();
            best = max(max(most[j & 1][0], most[j & 1][1]), max(most[j & 1][2], most[j & 1][3]));
          }
          last = best;
          if (threadIdx.x == 0) top[j] = best;
        }
      } else {
        for (int i = threadIdx.x; i < found; i += C::kThreads) {
          const uint64_t own_key = list[i];
          int above = 0;
          for (int j = 0; j < found; ++j) above += list[j] > own_key;
          if (above < top_k) top[above] = own_key;
        }
      }
      __syncthreads();
    }
    if (wave == 0) {
      if constexpr (W > 1) {
        s = (sums[0][0] + sums[0][1]) + (sums[0][2] + sums[0][3]);
        a = (sums[1][0] + sums[1][1]) + (sums[1][2] + sums[1][3]);
        eq = (sums[2][0] + sums[2][1]) + (sums[2][2] + sums[2][3]);
      }
      const Part p{m, m == -INFINITY ? 0.f : s + (eq - 1.f), a};
      if (parts == 1) {
        write_row(row, r, classes, labels, top_k, p, top, o);
      } else {
        const int64_t item = r * parts + blockIdx.x;
        if (lane == 0) part_out[item] = make_float4(p.m, p.t, p.a, 0.f);
        if (lane < top_k) keys_out[item * top_k + lane] = top[lane];
      }
    }
    __syncthreads();  // the next turn writes the LDS again
  }
}

// Joins the parts of a row, one wavefront per row.  Lane l takes the parts l,
// l + 64, ..; the best classes come off the heads of 63 of the parts' lists at
// a time and of the list so far (lane 63).
template <typename T>
__global__ __launch_bounds__(64) void k_scores_join(const T* __restrict__ z, int64_t ldz, int64_t n, int classes,
                                                    int parts, const int32_t* __restrict__ labels, int top_k,
                                                    Outputs o, const float4* __restrict__ part_in,
                                                    const uint64_t* __restrict__ keys_in) {
  __shared__ uint64_t top[kMaxTop];
  const int lane = threadIdx.x;
  for (int64_t r = blockIdx.x; r < n; r += gridDim.x) {
    Part p{-INFINITY, 0.f, 0.f};
    for (int c = lane; c < parts; c += 64) {
      const float4 q = part_in[r * parts + c];
      p = join(p, Part{q.x, q.y, q.z});
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const Part q{__shfl_xor(p.m, d, 64), __shfl_xor(p.t, d, 64), __shfl_xor(p.a, d, 64)};
      p = (lane & d) ? join(q, p) : join(p, q);  // the lower lane's part first: every lane the same
    }
    if (lane < kMaxTop) top[lane] = 0;
    __syncthreads();
    if (top_k > 0) {
      for (int c0 = 0; c0 < parts; c0 += 63) {
        const uint64_t* mine = keys_in + (r * parts + c0 + lane) * top_k;
        const bool have = lane < 63 && c0 + lane < parts;
        int at = 0;  // entries taken off this lane's list
        uint64_t keep = lane < top_k ? top[lane] : 0;  // the list so far
        uint64_t head = have ? mine[0] : lane == 63 ? top[0] : 0;
        __syncthreads();
        for (int j = 0; j < top_k; ++j) {
          const uint64_t win = wave_max_key(head);
          if (lane == 0) top[j] = win;
          const bool took = win != 0 && head == win;
          const bool old = __ballot(took) >> 63 & 1;  // off the list so far
          if (took) ++at;
          const int at63 = __shfl(at, 63, 64);
          const uint64_t next63 = (uint64_t)__shfl((uint32_t)(keep >> 32), at63 & 63, 64) << 32 |
                                  __shfl((uint32_t)keep, at63 & 63, 64);
          if (took && have) head = at < top_k ? mine[at] : 0;
          if (old && lane == 63) head = at63 < top_k ? next63 : 0;
        }
        __syncthreads();
      }
    }
    write_row(z + r * ldz, r, classes, labels, top_k, p, top, o);
    __syncthreads();
  }
}

// ------------------------------------------------------------- short rows
// One thread per row of at most NC classes, the row in its registers.  A
// wavefront reads 64 consecutive rows with 16-byte loads at each row's own
// alignment (the hardware takes any), a row's loads back to back so that the
// lines its lanes share are still in the L1.  The KT best are kept sorted by
// insertion, a strict comparison from the lowest class up (so ties stay in
// order); the first of them is the row's largest, left out of t.
// Values [AT, AT + N) of the row, N values of at most 16 bytes; -inf past the end.
template <typename T, int AT, int N, int NC>
__device__ __forceinline__ void load_span(const T* __restrict__ row, int classes, float (&x)[NC]) {
  if (AT + N <= classes) {
    if constexpr (N == 1) {
      x[AT] = ld(row + AT);
    } else {
      uint32_t w[N * sizeof(T) / 4];
      __builtin_memcpy(w, row + AT, N * sizeof(T));
#pragma unroll
      for (int i = 0; i < N; ++i)
        x[AT + i] = sizeof(T) == 4 ? __uint_as_float(w[i])
                    : i % 2        ? __uint_as_float(w[i / 2] & 0xffff0000u)
                                   : __uint_as_float(w[i / 2] << 16);
    }
  } else if constexpr (N > 1) {
    load_span<T, AT, N / 2>(row, classes, x);
    load_span<T, AT + N / 2, N / 2>(row, classes, x);
  } else {
    x[AT] = -INFINITY;
  }
}
template <typename T, int NC, int AT = 0>
__device__ __forceinline__ void load_row(const T* __restrict__ row, int classes, float (&x)[NC]) {
  constexpr int V = 16 / (int)sizeof(T);
  if constexpr (AT < NC) {
    load_span<T, AT, V>(row, classes, x);
    load_row<T, NC, AT + V>(row, classes, x);
  }
}

template <typename T, int NC, int KT>
__global__ __launch_bounds__(64) void k_scores_rows(const T* __restrict__ z, int64_t ldz, int64_t n, int classes,
                                                    const int32_t* __restrict__ labels, int top_k, Outputs o) {
  const int64_t r = (int64_t)blockIdx.x * 64 + threadIdx.x;
  if (r >= n) return;
  const T* row = z + r * ldz;
  float x[NC];
  load_row<T, NC>(row, classes, x);
  const int lab = o.logprob ? labels[r] : -1;
  float m = -INFINITY, tv[KT];
  int ti[KT];
#pragma unroll
  for (int j = 0; j < KT; ++j) {
    tv[j] = -INFINITY;
    ti[j] = -1;
  }
#pragma unroll
  for (int k0 = 0; k0 < NC; k0 += 4)
    if (k0 < classes) {
#pragma unroll
      for (int k = k0; k < k0 + 4; ++k) {
        const float v = x[k];  // -inf past the end: above nothing
        m = OpMax::of(m, v);
        bool above[KT];
#pragma unroll
        for (int j = 0; j < KT; ++j) above[j] = v > tv[j];
#pragma unroll
        for (int j = KT - 1; j >= 0; --j) {
          const int up = j > 0 ? j - 1 : 0;
          const bool shift = j > 0 && above[up];
          tv[j] = shift ? tv[up] : above[j] ? v : tv[j];
          ti[j] = shift ? ti[up] : above[j] ? k : ti[j];
        }
      }
    }
  Part p{m, 0.f, 0.f};
  const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
  for (int k0 = 0; k0 < NC; k0 += 4)
    if (k0 < classes) {
#pragma unroll
      for (int k = k0; k < k0 + 4; ++k) {
        // 2^h, as in k_scores_chunk
        const float h = fmaxf(k == ti[0] ? -INFINITY : (x[k] - base) * 1.44269504088896340736f, -300.f);
        const float e = __builtin_amdgcn_exp2f(h);
        p.t += e;
        p.a = fmaf(e, h, p.a);
      }
    }
  p.a *= 0.69314718055994530942f;
  const float2 lh = finish(p);
  if (o.logprob) o.logprob[r] = lab < 0 ? 0.f : lab >= classes ? NAN : (ld(row + lab) - base) - lh.x;
  o.entropy[r] = lh.y;
  reinterpret_cast<float2*>(o.stats)[r] = make_float2(m, lh.x);
  if (top_k == 0) return;
  if (m != m) {  // a NaN, which the comparisons passed over: one more pass per class
    uint64_t last = ~0ull;
    for (int j = 0; j < top_k; ++j) {
      uint64_t best = 0;
      for (int k = 0; k < classes; ++k) {
        const uint64_t key = rank_key(ld(row + k), (uint32_t)k);
        if (key < last && key > best) best = key;
      }
      last = best;
      o.top_index[r * top_k + j] = (int32_t)key_class(best);
      o.top_logprob[r * top_k + j] = NAN;
    }
    return;
  }
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
  int32_t* ix = o.top_index + r * top_k;
  float* lp = o.top_logprob + r * top_k;
  if (top_k == KT) {  // one wide store
#pragma unroll
    for (int j = 0; j < KT; ++j) ix[j] = ti[j];
#pragma unroll
    for (int j = 0; j < KT; ++j) lp[j] = (tv[j] - base) - lh.x;
  } else {
#pragma unroll
    for (int j = 0; j < KT; ++j)
      if (j < top_k) {
        ix[j] = ti[j];
        lp[j] = (tv[j] - base) - lh.x;
      }
  }
}

// Which kernel takes a row, by its length alone (and, for rows of several
// chunks, by how many there are): one workgroup holds up to 64 W E values.
struct Route {
  int waves, per_thread;  // W, E
  int parts;              // chunks of a row
};
Route route_of(int64_t n, int classes) {
  // up to 7 values of the first piece may belong to the row before
  const int64_t len = (int64_t)classes + 7;
  if (classes <= 510) return {1, 8, 1};     // 4-byte pieces: at most one such value
  if (len <= 2048) return {4, 8, 1};
  if (len <= 8192) return {4, 32, 1};
  // long rows: chunks of 8192 once they are enough workgroups for 256 CUs,
  // else four times as many
  const int64_t big = ceil_div(len, 8192);
  return n * big >= 512 ? Route{4, 32, (int)big} : Route{4, 8, (int)ceil_div(len, 2048)};
}

constexpr int kRowMax = 64;  // classes of a row that one thread takes

template <typename T, int NC>
void launch_rows(const T* z, int64_t ldz, int64_t n, int classes, const int32_t* labels, int top_k, const Outputs& o,
                 hipStream_t s) {
  const unsigned g = (unsigned)ceil_div(n, 64);
  if (top_k <= 1)
    k_scores_rows<T, NC, 1><<<g, 64, 0, s>>>(z, ldz, n, classes, labels, top_k, o);
  else if (top_k <= 3)
    k_scores_rows<T, NC, 3><<<g, 64, 0, s>>>(z, ldz, n, classes, labels, top_k, o);
  else if (top_k <= 8)
    k_scores_rows<T, NC, 8><<<g, 64, 0, s>>>(z, ldz, n, classes, labels, top_k, o);
  else
    k_scores_rows<T, NC, 16><<<g, 64, 0, s>>>(z, ldz, n, classes, labels, top_k, o);
}

template <typename T>
sscn_status launch_scores(const T* z, int64_t ldz, int64_t n, int classes, const int32_t* labels, int top_k,
                          const Outputs& o, void* workspace, hipStream_t s) {
  if (classes <= kRowMax) {
    if (classes <= 16)
      launch_rows<T, 16>(z, ldz, n, classes, labels, top_k, o, s);
    else if (classes <= 32)
      launch_rows<T, 32>(z, ldz, n, classes, labels, top_k, o, s);
    else
      launch_rows<T, 64>(z, ldz, n, classes, labels, top_k, o, s);
    SSCN_HIP(hipGetLastError());
    return SSCN_OK;
  }
  const Route w = route_of(n, classes);
  const int64_t items = n * w.parts;
  float4* parts = (float4*)workspace;
  uint64_t* keys = (uint64_t*)(parts + items);
  // a workgroup takes rows in turn once there are some 16384 of them
  const dim3 g((unsigned)w.parts, (unsigned)std::max<int64_t>(1, std::min<int64_t>(n, 16384 / w.parts)));
  if (w.waves == 1)
    k_scores_chunk<T, 1, 8><<<g, 64, 0, s>>>(z, ldz, n, classes, labels, top_k, o, parts, keys);
  else if (w.per_thread == 8)
    k_scores_chunk<T, 4, 8><<<g, 256, 0, s>>>(z, ldz, n, classes, labels, top_k, o, parts, keys);
  else
    k_scores_chunk<T, 4, 32><<<g, 256, 0, s>>>(z, ldz, n, classes, labels, top_k, o, parts, keys);
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
__device__ __forceinline__ GradRow grad_row(const GradInputs& q, int64_t r, int classes) {
  GradRow w;
  const float2 st = reinterpret_cast<const float2*>(q.stats)[r];
  w.L = st.y;
  w.empty = st.x == -INFINITY && st.y == 0.f;
  w.base = w.empty ? 0.f : st.x;
  w.h = q.dentropy ? q.dentropy[r] : 0.f;
  w.H = q.dentropy ? q.entropy[r] : 0.f;
  w.lab = q.dlogprob ? q.labels[r] : -1;
  w.g = w.lab < 0 ? 0.f : w.lab >= classes ? NAN : q.dlogprob[r];
  w.G = w.g;
  for (int j = 0; j < q.top_k; ++j) w.G += q.dtop[r * q.top_k + j];
  if (w.L != w.L) w.G = NAN;  // the clamp below would lose it
  if (w.empty) w.g = w.G = w.h = 0.f;
  return w;
}
__device__ __forceinline__ float grad_dense(const GradRow& w, float x) {
  const float lp = fmaxf((x - w.base) - w.L, -300.f);  // e^-300 is 0: no 0 * inf
  return -__builtin_amdgcn_exp2f(lp * 1.44269504088896340736f) * fmaf(w.h, lp + w.H, w.G);
}
__device__ __forceinline__ float grad_direct(const GradRow& w, float x, float A) {
  const float lp = (x - w.base) - w.L, p = expf(lp);
  return -A * expm1f(lp) - p * ((w.G - A) + (p == 0.f ? 0.f : w.h * (lp + w.H)));
}
// What class k receives directly.
__device__ __forceinline__ float direct_of(const GradInputs& q, const GradRow& w, int64_t r, int k) {
  float A = k == w.lab ? w.g : 0.f;
  for (int j = 0; j < q.top_k; ++j) A += q.top_index[r * q.top_k + j] == k ? q.dtop[r * q.top_k + j] : 0.f;
  return w.empty ? 0.f : A;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {  // nearest even, NaN kept
  typedef __bf16 B2 __attribute__((ext_vector_type(2)));
  typedef float F2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(F2{lo, hi}, B2));
}

// Short rows, a thread per row as in k_scores_rows.  The 64 rows of a
// wavefront go out through LDS, rows an odd number of words apart (each lane
// its own bank), as consecutive words of 4 bytes (WORDS) or single values.
template <typename T, int NC, bool WORDS>
__global__ __launch_bounds__(64) void k_grad_rows(const T* __restrict__ z, int64_t ldz, int64_t n, int classes,
                                                  GradInputs q, T* __restrict__ dz, int64_t ldd, int stride,
                                                  uint32_t magic) {
  extern __shared__ uint32_t lds[];
  const int64_t r0 = (int64_t)blockIdx.x * 64, r = r0 + threadIdx.x;
  T* out = reinterpret_cast<T*>(lds + threadIdx.x * stride);
  if (r < n) {
    const T* row = z + r * ldz;
    float x[NC];
    load_row<T, NC>(row, classes, x);
    const GradRow w = grad_row(q, r, classes);
#pragma unroll
    for (int k0 = 0; k0 < NC; k0 += 4)
      if (k0 < classes) {
#pragma unroll
        for (int k = k0; k < k0 + 4; ++k) x[k] = grad_dense(w, x[k]);
        // whole words: the stride has room for a last group's unused values
        if constexpr (sizeof(T) == 4) {
          __builtin_memcpy(out + k0, x + k0, 16);
        } else {
          const uint32_t v[2] = {pack_bf16(x[k0], x[k0 + 1]), pack_bf16(x[k0 + 2], x[k0 + 3])};
          __builtin_memcpy(out + k0, v, 8);
        }
      }
    if (w.lab >= 0 && w.lab < classes) st(out + w.lab, grad_direct(w, ld(row + w.lab), direct_of(q, w, r, w.lab)));
    for (int j = 0; j < q.top_k; ++j) {
      const int k = q.top_index[r * q.top_k + j];
      if (k >= 0 && k < classes) st(out + k, grad_direct(w, ld(row + k), direct_of(q, w, r, k)));
    }
  }
  __syncthreads();
  const int rows = (int)min<int64_t>(64, n - r0);
  const int per = WORDS ? classes * (int)sizeof(T) / 4 : classes;  // items of a row
  for (int i = threadIdx.x; i < rows * per; i += 64) {
    const int row = (int)(((uint32_t)i * magic) >> 20), at = i - row * per;  // i / per, exact for i < 4096
    T* to = dz + (r0 + row) * ldd;
    if constexpr (WORDS)
      reinterpret_cast<uint32_t*>(to)[at] = lds[row * stride + at];
    else
      to[at] = reinterpret_cast<const T*>(lds + row * stride)[at];
  }
}

// Longer rows, a chunk of a row per turn of a workgroup.
template <typename T, int W, int E>
__global__ __launch_bounds__(64 * W) void k_grad_chunk(const T* __restrict__ z, int64_t ldz, int64_t n, int classes,
                                                       int parts, GradInputs q, T* __restrict__ dz, int64_t ldd) {
  using C = Chunk<T, W, E>;
  const int64_t total = n * parts;
  for (int64_t item = blockIdx.x; item < total; item += gridDim.x) {
    const int64_t r = item / parts;
    const T* row = z + r * ldz;
    T* to = dz + r * ldd;
    const int64_t c0 = (item - r * parts) * C::kPieces * C::V - C::head(row);
    C chunk;
    chunk.load(row, classes, c0);
    const GradRow w = grad_row(q, r, classes);
#pragma unroll
    for (int g = 0; g < C::G; ++g) {
      float x[C::V];
#pragma unroll
      for (int i = 0; i < C::V; ++i) x[i] = grad_dense(w, chunk.at(g, i));
      const int64_t k0 = c0 + ((int64_t)g * C::kThreads + threadIdx.x) * C::V;
      if (k0 >= 0 && k0 + C::V <= classes) {  // one store, at whatever alignment it has
        if constexpr (sizeof(T) == 4) {
          __builtin_memcpy(to + k0, x, sizeof(T) * C::V);
        } else {
          uint32_t v[C::V / 2];
#pragma unroll
          for (int i = 0; i < C::V / 2; ++i) v[i] = pack_bf16(x[2 * i], x[2 * i + 1]);
          __builtin_memcpy(to + k0, v, sizeof(T) * C::V);
        }
      } else {
#pragma unroll
        for (int i = 0; i < C::V; ++i)
          if (k0 + i >= 0 && k0 + i < classes) st(to + k0 + i, x[i]);
      }
    }
    __syncthreads();  // the chunk's stores come before those below
    for (int j = threadIdx.x - 1; j < q.top_k; j += C::kThreads) {
      const int k = j < 0 ? w.lab : q.top_index[r * q.top_k + j];
      if (k >= 0 && k < classes && k >= c0 && k < c0 + C::kPieces * C::V)
        st(to + k, grad_direct(w, ld(row + k), direct_of(q, w, r, k)));
    }
  }
}

template <typename T, int NC>
void launch_grad_rows(const T* z, int64_t ldz, int64_t n, int classes, const GradInputs& q, T* dz, int64_t ldd,
                      hipStream_t s) {
  const int bytes = (int)sizeof(T) * classes;
  const bool words = bytes % 4 == 0 && ldd * sizeof(T) % 4 == 0 && reinterpret_cast<uintptr_t>(dz) % 4 == 0;
  const int stride = (int)(ceil_div(classes, 4) * 4 * sizeof(T) / 4) | 1;
  const int per = words ? bytes / 4 : classes;
  const uint32_t magic = ((1u << 20) + per - 1) / per;
  const unsigned g = (unsigned)ceil_div(n, 64);
  const size_t lds = (size_t)64 * stride * 4;
  if (words)
    k_grad_rows<T, NC, true><<<g, 64, lds, s>>>(z, ldz, n, classes, q, dz, ldd, stride, magic);
  else
    k_grad_rows<T, NC, false><<<g, 64, lds, s>>>(z, ldz, n, classes, q, dz, ldd, stride, magic);
}

template <typename T>
sscn_status launch_grad(const T* z, int64_t ldz, int64_t n, int classes, const GradInputs& q, T* dz, int64_t ldd,
                        hipStream_t s) {
  if (classes <= 16) {
    launch_grad_rows<T, 16>(z, ldz, n, classes, q, dz, ldd, s);
  } else if (classes <= 32) {
    launch_grad_rows<T, 32>(z, ldz, n, classes, q, dz, ldd, s);
  } else if (classes <= kRowMax) {
    launch_grad_rows<T, 64>(z, ldz, n, classes, q, dz, ldd, s);
  } else if (classes <= 510) {
    k_grad_chunk<T, 1, 8><<<(unsigned)std::min<int64_t>(n, 16384), 64, 0, s>>>(z, ldz, n, classes, 1, q, dz, ldd);
  } else {
    const int parts = (int)ceil_div((int64_t)classes + 7, 2048);
    k_grad_chunk<T, 4, 8><<<(unsigned)std::min<int64_t>(n * parts, 16384), 256, 0, s>>>(z, ldz, n, classes, parts, q,
                                                                                        dz, ldd);
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
  const GradInputs q{labels, stats, entropy, dtop ? top_k : 0, top_index, dlogprob, dentropy, dtop};
  return dtype == SSCN_F32 ? launch_grad((const float*)logits, ldz, n, classes, q, (float*)dlogits, ldd, stream)
                           : launch_grad((const uint16_t*)logits, ldz, n, classes, q, (uint16_t*)dlogits, ldd, stream);
}
