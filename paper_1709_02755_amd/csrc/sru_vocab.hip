// Rows of logits over a vocabulary: log probabilities of given tokens with
// entropy and top alternatives, distillation from a teacher's top logits, and
// their gradients.
//
// All of them need, of a row z of V logits at temperature T,
//   m = max z,  S = sum_j e^{x_j},  x_j = (z_j - m) / T  (and sum_j e^{x_j} x_j),
// taken in one pass with a running maximum, and then elementwise work.  They
// are bound by reading (and writing) the rows.
#include <math.h>

#include "sru_lanes.h"
#include "sru_lm.h"

namespace sru {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.693147180559945309f;
// 2^x is 0 in fp32 from here down: exponents are cut here where they are a
// factor, so that a probability of 0 times its log is 0 and not NaN (logits
// of -inf, or of the type's lowest value at a temperature below 1).
constexpr float kLowExp = -200.0f;

// Vectors that are not used again: past the caches, which keep what is (the
// second read of a row whose gradient is written: loss and gradient of 2048 x
// 131072 bf16 328 -> 263 us; the gradient alone of 4096 x 65536 270 -> 247).
typedef unsigned Quad __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load_last(const uint4* p) {
  const Quad q = __builtin_nontemporal_load(reinterpret_cast<const Quad*>(p));
  return make_uint4(q[0], q[1], q[2], q[3]);
}
__device__ __forceinline__ void store_last(uint4* p, const uint4& v) {
  const Quad q = {v.x, v.y, v.z, v.w};
  __builtin_nontemporal_store(q, reinterpret_cast<Quad*>(p));
}

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

template <bool BF16>
struct Elem;
template <>
struct Elem<false> {
  using T = float;
  static constexpr int VE = 4;  // elements of a 16-byte vector
  static __device__ __forceinline__ float get(float v) { return v; }
  static __device__ __forceinline__ float put(float v) { return v; }
  static __device__ __forceinline__ void unpack(const uint4& u, float (&f)[4]) {
    f[0] = __uint_as_float(u.x);
    f[1] = __uint_as_float(u.y);
    f[2] = __uint_as_float(u.z);
    f[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[4]) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]),
                      __float_as_uint(f[3]));
  }
  static constexpr unsigned kNegInf = 0xff800000u;
};
template <>
struct Elem<true> {
  using T = uint16_t;
  static constexpr int VE = 8;
  static __device__ __forceinline__ float get(uint16_t v) {
    return __uint_as_float((unsigned)v << 16);
  }
  static __device__ __forceinline__ uint16_t put(float v) {
    return __builtin_bit_cast(uint16_t, (__bf16)v);
  }
  static __device__ __forceinline__ void unpack(const uint4& u, float (&f)[8]) {
    const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float (&f)[8]) {
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = (unsigned)put(f[2 * i]) | ((unsigned)put(f[2 * i + 1]) << 16);
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
  static constexpr unsigned kNegInf = 0xff80ff80u;
};

// How a row is cut: up to the first 16-byte boundary, whole vectors, the rest.
// A part of a row is a range of its vectors; the first part takes the head
// and the last one the tail as well.
struct Span {
  int head, nvec, tail;
};
template <bool BF16>
__device__ __forceinline__ Span row_span(const typename Elem<BF16>::T* z, int V) {
  constexpr int ES = sizeof(typename Elem<BF16>::T), VE = Elem<BF16>::VE;
  const int mis = (int)(reinterpret_cast<uintptr_t>(z) & 15);
  Span s;
  s.head = min(V, ((16 - mis) & 15) / ES);
  s.nvec = (V - s.head) / VE;
  s.tail = s.head + s.nvec * VE;
  return s;
}

// ------------------------------------------------------- running statistics
// Maximum m, s = sum 2^x and t = sum 2^x x with x = (z - m) k, k = log2(e) / T.
// base is m, or 0 while there is nothing above -inf (z - base is then -inf and
// adds 0, where z - m would be NaN).  A NaN or +inf makes s NaN.
template <bool ENT>
struct Run {
  float m = -INFINITY, base = 0.f, s = 0.f, t = 0.f;

  // brings (s, t) to the maximum nm >= m
  __device__ __forceinline__ void to(float nm, float k) {
    // m = -inf: nothing was added, and nothing is scaled
    const float d = m == -INFINITY ? 0.f : fmaxf((m - nm) * k, kLowExp);
    const float f = m == nm ? 1.f : exp2_hw(d);
    if constexpr (ENT) t = m == nm ? t : f * (t + d * s);
    s *= f;
    m = nm;
    base = nm == -INFINITY ? 0.f : nm;
  }
  template <int VE>
  __device__ __forceinline__ void add(const float (&z)[VE], float vmax, float k) {
    if (vmax > m) to(vmax, k);
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      const float x = (z[j] - base) * k;
      const float e = exp2_hw(x);
      s += e;
      if constexpr (ENT) t = fmaf(e, fmaxf(x, kLowExp), t);
    }
  }
};

template <bool ENT>
__device__ __forceinline__ void run_store(float* p, const Run<ENT>& r) {
  p[0] = r.m;
  p[1] = r.s;
  p[2] = r.t;
}
template <bool ENT>
__device__ __forceinline__ Run<ENT> run_load(const float* p) {
  Run<ENT> r;
  r.m = p[0];
  r.base = r.m == -INFINITY ? 0.f : r.m;
  r.s = p[1];
  r.t = p[2];
  return r;
}

// The statistics of a workgroup's threads, the same in every thread; always in
// the same order.  lds: 3 floats a wave; barriers inside.
template <int LANES, bool ENT>
__device__ __forceinline__ void run_lanes(Run<ENT>& r, float k) {
  r.to(lanes_max<LANES>(r.m), k);
  r.s = lanes_sum<LANES>(r.s);
  if constexpr (ENT) r.t = lanes_sum<LANES>(r.t);
}
template <int THREADS, bool ENT>
__device__ __forceinline__ Run<ENT> run_block(Run<ENT> r, float k, float* lds) {
  run_lanes<64>(r, k);
  constexpr int W = THREADS / 64;
  if ((threadIdx.x & 63) == 0) run_store(lds + 3 * (threadIdx.x >> 6), r);
  __syncthreads();
  r = run_load<ENT>(lds + 3 * (threadIdx.x & (W - 1)));
  run_lanes<W>(r, k);
  __syncthreads();
  return r;
}

// ---------------------------------------------------------- top alternatives
// Values are ordered by an unsigned key (larger = better), equal ones by the
// lower column; -0 counts as 0, and a NaN is no alternative.
__device__ __forceinline__ unsigned top_key(float z) {
  const unsigned u = __float_as_uint(z + 0.0f);
  return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float top_value(unsigned key) {
  return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ bool top_better(unsigned k, unsigned i, unsigned k2, unsigned i2) {
  return k > k2 || (k == k2 && i < i2);
}

// A wave's 64 keys, the largest in lane 0: runs of SIZE lanes are sorted from two
// of half the size, first against each other's mirror image.
template <int O>
__device__ __forceinline__ unsigned sort_step(unsigned key) {
  constexpr int high = O > 31 ? 32 : O > 15 ? 16 : O > 7 ? 8 : O > 3 ? 4 : O > 1 ? 2 : 1;
  const unsigned o = lane_xor<O>(key);
  return threadIdx.x & high ? min(key, o) : max(key, o);
}
template <int STEP>
__device__ __forceinline__ unsigned sort_steps(unsigned key) {
  if constexpr (STEP > 0) return sort_steps<STEP / 2>(sort_step<STEP>(key));
  return key;
}
template <int SIZE = 64>
__device__ __forceinline__ unsigned wave_sort(unsigned key) {
  if constexpr (SIZE > 2) key = wave_sort<SIZE / 2>(key);
  return sort_steps<SIZE / 4>(sort_step<SIZE - 1>(key));
}

// Candidates for a row's best K, found by one of a workgroup's W waves: in its
// LDS, unsorted, all that may be among them.  Mostly few are found: the lanes'
// best values so far bound them from below (K of a wave's lanes have a value as
// good as the K-th best of these; so have K / W lanes of every wave, by the
// least of the waves' K / W-th best), and the bounds are taken anew whenever
// twice as much has been read.  Where the list fills up all the same (values
// that rise along the row, or are all alike) it is cut to its best K.
constexpr int kFoundRest = 128;  // room beyond the candidates of one load
template <int W>
struct Found {
  uint2* list;
  unsigned* floor;   // LDS, one word for the workgroup: K values have this key or a better one
  unsigned* bounds;  // LDS, a word for each wave
  int K;
  int n = 0;
  unsigned tk = 0, ti = 0xffffffffu;  // the K-th entry when the list was cut last
  unsigned best = 0;                  // this lane's best key

  __device__ __forceinline__ void raise(unsigned key) {
    if ((threadIdx.x & 63) == 0 && key) atomicMax(floor, key);
  }
  // by all waves together
  __device__ __forceinline__ void bound() {
    const unsigned sorted = wave_sort(best);
    if ((threadIdx.x & 63) == 0)
      bounds[threadIdx.x >> 6] = __builtin_amdgcn_readlane(sorted, (K - 1) / W);
    raise(__builtin_amdgcn_readlane(sorted, K - 1));
    __syncthreads();
    unsigned least = bounds[0];
#pragma unroll
    for (int w = 1; w < W; ++w) least = min(least, bounds[w]);
    raise(least);
    __syncthreads();
  }

  // values f of columns col .. (none where col is past V)
  template <int VE>
  __device__ __forceinline__ void take(const float (&f)[VE], float vmax, unsigned col, unsigned V) {
    const unsigned shared = *(volatile unsigned*)floor;
    if (!__any(top_key(vmax) >= max(tk, shared))) return;
#pragma unroll
    for (int j = 0; j < VE; ++j) {
      const unsigned key = top_key(f[j]), at = col + j;
      const bool ok = f[j] == f[j] && key >= shared && at < V && top_better(key, at, tk, ti);
      const unsigned long long b = __ballot(ok);
      if (ok)
        list[n + __builtin_amdgcn_mbcnt_hi((unsigned)(b >> 32),
                                           __builtin_amdgcn_mbcnt_lo((unsigned)b, 0))] =
            make_uint2(key, at);
      n += __popcll(b);
    }
    if (n > kFoundRest) cut();
  }
  __device__ __forceinline__ void cut() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int lane = threadIdx.x & 63;
    for (int e = 0; e < n; e += 64) {
      const uint2 x = list[min(e + lane, n - 1)];
      int rank = 0;
      for (int i = 0; i < n; ++i) {
        const uint2 y = list[i];
        rank += top_better(y.x, y.y, x.x, x.y);
      }
      const unsigned long long b = __ballot(e + lane < n && rank == K - 1);
      if (b) {
        tk = __builtin_amdgcn_readlane(x.x, __ffsll((long long)b) - 1);
        ti = __builtin_amdgcn_readlane(x.y, __ffsll((long long)b) - 1);
      }
    }
    int kept = 0;
    for (int e = 0; e < n; e += 64) {
      const uint2 x = list[min(e + lane, n - 1)];
      const bool ok = e + lane < n && !top_better(tk, ti, x.x, x.y);
      const unsigned long long b = __ballot(ok);
      // at or before the place it was read from, which the wave is past
      if (ok)
        list[kept + __builtin_amdgcn_mbcnt_hi((unsigned)(b >> 32),
                                              __builtin_amdgcn_mbcnt_lo((unsigned)b, 0))] = x;
      kept += __popcll(b);
    }
    n = kept;
    raise(tk);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
};

// -------------------------------------------------------------- one row part
// Statistics of a part of a row, and the wave's candidates for its alternatives.
template <bool BF16, int THREADS, int U, bool ENT, bool TOP>
__device__ __forceinline__ Run<ENT> part_stats(const typename Elem<BF16>::T* z, int V, int part,
                                               int parts, float k,
                                               Found<THREADS / 64>& top) {
  using E = Elem<BF16>;
  constexpr int VE = E::VE;
  const Span sp = row_span<BF16>(z, V);
  const int tid = threadIdx.x;
  const int v0 = (int)((long long)sp.nvec * part / parts);
  const int v1 = (int)((long long)sp.nvec * (part + 1) / parts);
  const uint4* zv = reinterpret_cast<const uint4*>(z + sp.head);
  Run<ENT> run;

  auto largest = [](const float(&f)[VE]) {
    float vm = f[0];
#pragma unroll
    for (int j = 1; j < VE; ++j) vm = fmaxf(vm, f[j]);
    return vm;
  };
  auto take = [&](const float(&f)[VE], float vm, unsigned col) {
    run.add(f, vm, k);
    if constexpr (TOP) top.take(f, vm, col, (unsigned)V);
  };

  int again = 1;  // rounds until the bounds are taken anew
  for (int v = v0; v < v1; v += THREADS * U) {
    uint4 u[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int at = v + i * THREADS + tid;
      u[i] = make_uint4(E::kNegInf, E::kNegInf, E::kNegInf, E::kNegInf);
      if (at < v1) u[i] = zv[at];
    }
    float vm[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      float f[VE];
      E::unpack(u[i], f);
      vm[i] = largest(f);
      // (a NaN among others does not show in their largest, and alone is none)
      if (TOP && v + i * THREADS + tid < v1 && vm[i] == vm[i])
        top.best = max(top.best, top_key(vm[i]));
    }
    if (TOP && --again == 0) {
      top.bound();
      again = (v - v0) / (THREADS * U) + 1;
    }
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int at = v + i * THREADS + tid;
      float f[VE];
      E::unpack(u[i], f);
      take(f, vm[i], at < v1 ? (unsigned)(sp.head + at * VE) : 0x80000000u);
    }
  }
  // the head and the tail, at most VE - 1 elements each, one a lane
  int col = -1;
  if (part == 0 && tid < sp.head) col = tid;
  if (part == parts - 1 && tid >= 32 && tid - 32 < V - sp.tail) col = sp.tail + tid - 32;
  if (tid < 64) {
    float f[VE];
#pragma unroll
    for (int j = 0; j < VE; ++j) f[j] = -INFINITY;
    if (col >= 0) f[0] = E::get(z[col]);
    const float vm = f[0];
    run.add(f, vm, k);
    if constexpr (TOP) {
      // the other places of the vector are no columns
#pragma unroll
      for (int j = 1; j < VE; ++j) f[j] = NAN;
      top.take(f, vm, col >= 0 ? (unsigned)col : 0x80000000u, (unsigned)V);
    }
  }
  return run;
}

// The best K of several lists, n[l] entries in list l (of pitch `pitch`), in
// order: put(rank, key, column) for each, and for the places that nothing fills
// (key 0).  What is below the last bound is dropped first
// (into `kept`, LDS, at most `room` entries; with more, all are ranked).
template <int THREADS, typename F>
__device__ __forceinline__ void top_merge(const uint2* lists, int pitch, int count, const int* n,
                                          unsigned floor, int K, uint2* kept, int room,
                                          int* kept_n, F put) {
  int total = 0;
  for (int l = 0; l < count; ++l) total += n[l];
  if (threadIdx.x == 0) *kept_n = 0;
  __syncthreads();
  for (int e = threadIdx.x; e < total; e += THREADS) {
    int w = 0, i = e;
    while (i >= n[w]) i -= n[w++];
    const uint2 x = lists[w * pitch + i];
    if (x.x < floor) continue;  // K others are better
    const int to = atomicAdd(kept_n, 1);
    if (to < room) kept[to] = x;
  }
  __syncthreads();
  const int some = *kept_n;
  if (some <= room) {
    // in any order: a rank depends on the entries alone
    for (int e = threadIdx.x; e < some; e += THREADS) {
      const uint2 x = kept[e];
      int rank = 0;
      for (int i = 0; i < some; ++i) rank += top_better(kept[i].x, kept[i].y, x.x, x.y);
      if (rank < K) put(rank, x.x, x.y);
    }
  } else {
    for (int e = threadIdx.x; e < total; e += THREADS) {
      int w = 0, i = e;
      while (i >= n[w]) i -= n[w++];
      const uint2 x = lists[w * pitch + i];
      int rank = 0;
      for (int l = 0; l < count && rank < K; ++l)
        for (int q = 0; q < n[l]; ++q) {
          const uint2 y = lists[l * pitch + q];
          rank += top_better(y.x, y.y, x.x, x.y);
        }
      if (rank < K) put(rank, x.x, x.y);
    }
  }
  for (int r = total + threadIdx.x; r < K; r += THREADS) put(r, 0u, 0xffffffffu);
}

struct RowStats {
  float m, base, s, log_s;
};
__device__ __forceinline__ RowStats row_stats(float m, float s) {
  return RowStats{m, m == -INFINITY ? 0.f : m, s, logf(s)};
}
// log probability of a logit; a row with no logit above -inf gives -inf
__device__ __forceinline__ float row_logprob(const RowStats& r, float z, float inv_t) {
  return r.s == 0.f ? -INFINITY : (z - r.base) * inv_t - r.log_s;
}

// ------------------------------------------------- token log probabilities
// The row's token and its logit: asked for before the row is read, and while its
// sums are joined.
template <bool BF16>
struct Scored {
  int64_t tok;
  float z = 0.f;
  bool inside = false;
  __device__ __forceinline__ Scored(const LogprobArgs& a, int row) : tok(a.tokens[row]) {}
  __device__ __forceinline__ void gather(const LogprobArgs& a,
                                         const typename Elem<BF16>::T* row) {
    inside = tok >= 0 && tok < a.r.V;
    if (inside) z = Elem<BF16>::get(row[tok]);
  }
};
template <bool BF16>
__device__ __forceinline__ void logprob_write(const LogprobArgs& a, int row, float m, float s,
                                              float t, float inv_t, const Scored<BF16>& token) {
  const RowStats st = row_stats(m, s);
  a.stats[2LL * row] = m;
  a.stats[2LL * row + 1] = s;
  // H = log S - sum e^x x / S (t is in units of log 2); 0 where nothing is possible
  a.entropy[row] = s == 0.f ? 0.f : st.log_s - kLn2 * t / s;
  a.logprob[row] = token.inside ? row_logprob(st, token.z, inv_t) : 0.f;
}

__device__ __forceinline__ void top_write(const LogprobArgs& a, int row, const RowStats& st,
                                          float inv_t, int rank, unsigned key, unsigned idx) {
  const long long o = (long long)row * a.top + rank;
  a.top_ids[o] = key ? (int64_t)idx : -1;
  a.top_logprobs[o] = key ? row_logprob(st, top_value(key), inv_t) : -INFINITY;
}

// One part of one row per workgroup.  parts == 1: the row's results; else its
// statistics and its best alternatives go to the workspace, [row, part] of 4
// floats, then [row, part, K] pairs.
//
// Without alternatives it reads at 4.9 TB/s (2048 x 65536 bf16, 54 us) and is
// bound by that.  With alternatives, 1000 x 30011 fp32 takes 31, 34, 39 and 45 us for
// 1, 5, 20 and 64 of them, and 27 without: what passes the bounds is collected, cut
// and ranked by all rows at about the same time.  The bounds after the first round
// cost less than 1 us of that and save more (without them 31, 37, 48 and 130).
// Twenty of 4 x 131072 bf16, in eight parts a row, take 11.4 us and 6.7 to join:
// launches and waits, one after the other.  Loads a round ahead were slower in every
// case (1000 x 30011 26 -> 27 us, with alternatives 39 -> 52).
// Six waves on a SIMD rather than the five that the compiler would leave: three
// workgroups fit a CU (4096 x 32768 bf16, five alternatives, 90 -> 80 us).
template <bool BF16, int THREADS, int U, bool TOP>
__global__ __launch_bounds__(THREADS, TOP && BF16 ? 6 : 1) void logprob_kernel(LogprobArgs a, int parts) {
  using E = Elem<BF16>;
  constexpr int W = THREADS / 64, kPitch = 64 * E::VE + kFoundRest;
  __shared__ float red[3 * W];
  constexpr int kRoom = TOP ? 512 : 1;
  __shared__ unsigned floor, bounds[W];
  __shared__ int count[W], kept_n;
  __shared__ uint2 lists[TOP ? W * kPitch : 1], kept[kRoom];
  const int wave = threadIdx.x >> 6;
  const float inv_t = 1.f / a.r.temperature, k = kLog2e / a.r.temperature;
  const long long items = (long long)a.r.N * parts;
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    const int row = (int)(it / parts), part = (int)(it - (long long)row * parts);
    const auto* z = static_cast<const typename E::T*>(a.r.z) + (long long)row * a.r.ld;
    Scored<BF16> token(a, row);
    Found<W> top{lists + (TOP ? wave * kPitch : 0), &floor, bounds, a.top};
    if constexpr (TOP) {
      if (threadIdx.x == 0) floor = 0;
      __syncthreads();
    }
    Run<true> run = part_stats<BF16, THREADS, U, true, TOP>(z, a.r.V, part, parts, k, top);
    if (parts == 1) token.gather(a, z);
    if constexpr (TOP) {
      if ((threadIdx.x & 63) == 0) count[wave] = top.n;
    }
    run = run_block<THREADS>(run, k, red);  // its barriers make the lists visible
    if (parts == 1) {
      if (threadIdx.x == 0) logprob_write<BF16>(a, row, run.m, run.s, run.t, inv_t, token);
      if constexpr (TOP) {
        const RowStats st = row_stats(run.m, run.s);
        top_merge<THREADS>(lists, kPitch, W, count, floor, a.top, kept, kRoom, &kept_n,
                           [&](int rank, unsigned key, unsigned idx) {
                             top_write(a, row, st, inv_t, rank, key, idx);
                           });
      }
    } else {
      float* ws = static_cast<float*>(a.workspace);
      if (threadIdx.x == 0) run_store(ws + 4 * it, run);
      if constexpr (TOP) {
        uint2* wl = reinterpret_cast<uint2*>(ws + 4 * items) + it * a.top;
        top_merge<THREADS>(lists, kPitch, W, count, floor, a.top, kept, kRoom, &kept_n,
                           [&](int rank, unsigned key, unsigned idx) {
                             wl[rank] = make_uint2(key, idx);
                           });
      }
    }
    __syncthreads();  // lists, count and floor are used again
  }
}

constexpr int kMaxParts = 64;

// The parts of a row joined, one workgroup per row.
template <bool BF16, bool TOP>
__global__ __launch_bounds__(256) void logprob_join_kernel(LogprobArgs a, int parts) {
  extern __shared__ uint2 lists[];
  __shared__ int n[kMaxParts], kept_n;
  __shared__ unsigned floor;
  constexpr int kRoom = TOP ? 512 : 1;
  __shared__ uint2 kept[kRoom];
  const float inv_t = 1.f / a.r.temperature, k = kLog2e / a.r.temperature;
  const float* ws = static_cast<const float*>(a.workspace);
  const uint2* wl = reinterpret_cast<const uint2*>(ws + 4LL * a.r.N * parts);
  const int lane = threadIdx.x & 63;
  for (int row = blockIdx.x; row < a.r.N; row += gridDim.x) {
    if constexpr (TOP) {
      __syncthreads();  // the lists' earlier use
      for (int e = threadIdx.x; e < parts * a.top; e += 256)
        lists[e] = wl[(long long)row * parts * a.top + e];
    }
    // one part a lane, joined across the wave; every wave does the same
    Scored<BF16> token(a, row);
    Run<true> run;
    if (lane < parts) run = run_load<true>(ws + 4 * ((long long)row * parts + lane));
    token.gather(a, static_cast<const typename Elem<BF16>::T*>(a.r.z) + (long long)row * a.r.ld);
    run_lanes<64>(run, k);
    if (threadIdx.x == 0) logprob_write<BF16>(a, row, run.m, run.s, run.t, inv_t, token);
    if constexpr (TOP) {
      // K / parts entries of every list are at least as good as the least of the
      // lists' K / parts-th
      if (threadIdx.x == 0) floor = 0xffffffffu;
      __syncthreads();
      if (threadIdx.x < parts) {
        const uint2* l = lists + threadIdx.x * a.top;
        int filled = a.top;
        while (filled > 0 && l[filled - 1].x == 0) --filled;
        n[threadIdx.x] = filled;
        atomicMin(&floor, l[(a.top - 1) / parts].x);
      }
      __syncthreads();
      const RowStats st = row_stats(run.m, run.s);
      top_merge<256>(lists, a.top, parts, n, floor, a.top, kept, kRoom, &kept_n,
                     [&](int rank, unsigned key, unsigned idx) {
                       top_write(a, row, st, inv_t, rank, key, idx);
                     });
    }
  }
}

// ------------------------------------------------------------------ gradients
// dz_j = e_j (c0 + c1 x_j), e_j = 2^{x_j}, over a part of a row.  The first round
// of loads is made when the object is, ahead of what the gradient waits for.
template <bool BF16, int THREADS, int U>
struct PartGrad {
  using E = Elem<BF16>;
  static constexpr int VE = E::VE;
  const typename E::T* z;
  Span sp;
  int V, v0, v1;
  bool first, last;  // the part has the row's head, tail
  uint4 u[U];

  __device__ __forceinline__ void load(int v) {
    const uint4* zv = reinterpret_cast<const uint4*>(z + sp.head);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int at = v + i * THREADS + (int)threadIdx.x;
      if (at < v1) u[i] = load_last(zv + at);
    }
  }
  __device__ __forceinline__ PartGrad(const typename E::T* z_, int V_, int part, int parts)
      : z(z_), sp(row_span<BF16>(z_, V_)), V(V_), first(part == 0), last(part == parts - 1) {
    v0 = (int)((long long)sp.nvec * part / parts);
    v1 = (int)((long long)sp.nvec * (part + 1) / parts);
    load(v0);
  }
  template <bool LIN>
  __device__ __forceinline__ void write(typename E::T* dz, float base, float k, float c0,
                                        float c1) {
    const int tid = threadIdx.x;
    uint4* dv = reinterpret_cast<uint4*>(dz + sp.head);
    // rows of another alignment than their logits' are written element by element
    const bool whole = ((reinterpret_cast<uintptr_t>(dv)) & 15) == 0;
    // a row that adds nothing: exact zeros, whatever its logits are
    const bool none = c0 == 0.f && c1 == 0.f;
    auto grad = [&](float zj) {
      const float x = (zj - base) * k;
      const float e = exp2_hw(x);
      return none ? 0.f : LIN ? e * fmaf(c1, fmaxf(x, kLowExp), c0) : e * c0;
    };
    for (int v = v0; v < v1; v += THREADS * U) {
      if (v > v0 && !none) load(v);
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int at = v + i * THREADS + tid;
        if (at < v1) {
          float f[VE];
          E::unpack(u[i], f);
#pragma unroll
          for (int j = 0; j < VE; ++j) f[j] = grad(f[j]);
          if (whole) {
            store_last(dv + at, E::pack(f));
          } else {
#pragma unroll
            for (int j = 0; j < VE; ++j) dz[sp.head + at * VE + j] = E::put(f[j]);
          }
        }
      }
    }
    if (first && tid < sp.head) dz[tid] = E::put(grad(E::get(z[tid])));
    if (last && tid < V - sp.tail) dz[sp.tail + tid] = E::put(grad(E::get(z[sp.tail + tid])));
  }
};

// Whether column col lies in this part of the row.
template <bool BF16>
__device__ __forceinline__ bool in_part(const typename Elem<BF16>::T* z, int V, int col, int part,
                                        int parts) {
  constexpr int VE = Elem<BF16>::VE;
  const Span sp = row_span<BF16>(z, V);
  if (col < sp.head) return part == 0;
  if (col >= sp.tail) return part == parts - 1;
  const int v = (col - sp.head) / VE;
  const int v0 = (int)((long long)sp.nvec * part / parts);
  const int v1 = (int)((long long)sp.nvec * (part + 1) / parts);
  return v >= v0 && v < v1;
}

// The columns with a term of their own: n (column, weight) pairs in LDS,
// column -1 = none.  Entry e of the n belongs to thread e % THREADS; where a
// column occurs more than once its first entry adds all of them.  Before the
// part's gradient is written, each owner takes its logit; dz may be z.
template <bool BF16, int THREADS, int MAXN, bool LIN>
struct PointTerms {
  static constexpr int PER = (MAXN + THREADS - 1) / THREADS;
  using E = Elem<BF16>;
  float value[PER];
  int at[PER];
  // logits: of the columns, or nullptr: read from z
  __device__ __forceinline__ void take(const int* cols, const float* w, const float* logits, int n,
                                       const typename E::T* z, int V, int part, int parts,
                                       float base, float k, float c0, float c1) {
    const bool none = c0 == 0.f && c1 == 0.f;
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int e = p * THREADS + (int)threadIdx.x;
      at[p] = -1;
      if (e >= n) continue;
      const int c = cols[e];
      if (c < 0 || !in_part<BF16>(z, V, c, part, parts)) continue;
      float sum = 0.f;
      int first = e;
      for (int q = 0; q < n; ++q)
        if (cols[q] == c) {
          first = min(first, q);
          sum += w[q];
        }
      if (first != e) continue;
      const float x = ((logits ? logits[e] : E::get(z[c])) - base) * k;
      const float g = none ? 0.f
                           : exp2_hw(x) * (LIN ? fmaf(c1, fmaxf(x, kLowExp), c0) : c0);
      value[p] = g + sum;
      at[p] = c;
    }
  }
  __device__ __forceinline__ void put(typename E::T* dz) {
#pragma unroll
    for (int p = 0; p < PER; ++p)
      if (at[p] >= 0) dz[at[p]] = E::put(value[p]);
  }
};

// dz_j = (1/T) (w_t [j = t] + sum_k w_k [j = id_k] - p_j A - dH p_j (log p_j + H)),
// A = w_t + sum_k w_k, with p = e / S and log p = x ln2 - log S.
// Bound by memory: 2048 x 65536 bf16 in 85 us, 268 MB read (partly from the caches,
// after the forward) and as many written.
template <bool BF16, int THREADS, int U>
__global__ __launch_bounds__(THREADS) void logprob_grad_kernel(LogprobGradArgs a, int parts) {
  using E = Elem<BF16>;
  __shared__ int cols[kMaxTop + 1];
  __shared__ float wts[kMaxTop + 1];
  const float inv_t = 1.f / a.r.temperature, k = kLog2e / a.r.temperature;
  const int n = 1 + (a.dtop ? a.top : 0);
  const long long items = (long long)a.r.N * parts;
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    const int row = (int)(it / parts), part = (int)(it - (long long)row * parts);
    const auto* z = static_cast<const typename E::T*>(a.r.z) + (long long)row * a.r.ld;
    auto* dz = static_cast<typename E::T*>(a.dz) + (long long)row * a.ldd;
    const float s = a.stats[2LL * row + 1];
    const RowStats st = row_stats(a.stats[2LL * row], s);
    PartGrad<BF16, THREADS, U> pg(z, a.r.V, part, parts);
    for (int e = threadIdx.x; e < n; e += THREADS) {
      const int64_t c = e == 0 ? (a.dlogprob ? a.tokens[row] : -1)
                               : a.top_ids[(long long)row * a.top + e - 1];
      const bool live = c >= 0 && c < a.r.V && s != 0.f;
      cols[e] = live ? (int)c : -1;
      wts[e] = !live ? 0.f
                     : inv_t * (e == 0 ? a.dlogprob[row] : a.dtop[(long long)row * a.top + e - 1]);
    }
    __syncthreads();
    float sum = 0.f;
    for (int e = 0; e < n; ++e) sum += wts[e];
    const float inv_s = s == 0.f ? 0.f : 1.f / s;
    const float dh = a.dentropy && s != 0.f ? a.dentropy[row] * inv_t : 0.f;
    const float c0 = -(sum + (dh == 0.f ? 0.f : dh * (a.entropy[row] - st.log_s))) * inv_s;
    const float c1 = dh == 0.f ? 0.f : -dh * kLn2 * inv_s;
    PointTerms<BF16, THREADS, kMaxTop + 1, true> pt;
    pt.take(cols, wts, nullptr, n, z, a.r.V, part, parts, st.base, k, c0, c1);
    __syncthreads();  // dz may be z
    if (c1 == 0.f)
      pg.template write<false>(dz, st.base, k, c0, 0.f);
    else
      pg.template write<true>(dz, st.base, k, c0, c1);
    __syncthreads();
    pt.put(dz);
    __syncthreads();
  }
}

// ------------------------------------------------------------------ distillation
// A row's teacher entries, thread e's every THREADS-th from e: fetched before the
// row is read, so that the student's logits of the ids can be asked for as soon
// as that has been (an id that is not kept has column -1).
template <bool BF16, int THREADS>
struct Teacher {
  static constexpr int PER = kMaxTeacher / THREADS;
  int64_t id[PER];
  float t[PER], z[PER];
  int col[PER];
  __device__ __forceinline__ void fetch(const DistillArgs& a, int row) {
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int e = p * THREADS + (int)threadIdx.x;
      if (e >= a.K) break;
      const long long o = (long long)row * a.K + e;
      id[p] = a.ids[o];
      t[p] = a.teacher_bf16 ? Elem<true>::get(static_cast<const uint16_t*>(a.teacher)[o])
                            : static_cast<const float*>(a.teacher)[o];
    }
  }
  __device__ __forceinline__ void gather(const DistillArgs& a, const typename Elem<BF16>::T* row) {
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int e = p * THREADS + (int)threadIdx.x;
      if (e >= a.K) break;
      const bool kept = id[p] >= 0 && id[p] < a.r.V && t[p] != -INFINITY;
      col[p] = kept ? (int)id[p] : -1;
      z[p] = kept ? Elem<BF16>::get(row[col[p]]) : 0.f;
    }
  }
  // The teacher's probabilities p = softmax(t / T) over the kept entries: cols,
  // probs, zs in LDS; returns 1 where there is any, else 0.  scratch: THREADS /
  // 64 floats.
  __device__ __forceinline__ float probabilities(const DistillArgs& a, int* cols, float* probs,
                                                 float* zs, float* scratch, float k) {
    constexpr int W = THREADS / 64;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float m = -INFINITY;
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int e = p * THREADS + (int)threadIdx.x;
      // a NaN that fmaxf drops comes back in the sum
      if (e < a.K && col[p] >= 0) m = fmaxf(m, t[p]);
    }
    m = lanes_max<64>(m);
    if (lane == 0) scratch[wave] = m;
    __syncthreads();
    for (int w = 0; w < W; ++w) m = fmaxf(m, scratch[w]);
    __syncthreads();
    float s = 0.f;
    bool any = false;
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int e = p * THREADS + (int)threadIdx.x;
      if (e >= a.K) break;
      t[p] = col[p] >= 0 ? exp2_hw((t[p] - m) * k) : 0.f;
      s += t[p];
      any |= col[p] >= 0;
    }
    s = lanes_sum<64>(s);
    if (lane == 0) scratch[wave] = s;
    const int some = __syncthreads_or(any);
    s = 0.f;
    for (int w = 0; w < W; ++w) s += scratch[w];
    const float inv = 1.f / s;
#pragma unroll
    for (int p = 0; p < PER; ++p) {
      const int e = p * THREADS + (int)threadIdx.x;
      if (e >= a.K) break;
      cols[e] = col[p];
      probs[e] = col[p] >= 0 ? t[p] * inv : 0.f;
      zs[e] = z[p];
    }
    __syncthreads();
    return some ? 1.f : 0.f;
  }
};

// sum p (log p - log q) over the kept entries with p > 0, in every thread
template <int THREADS>
__device__ __forceinline__ float distill_loss(const DistillArgs& a, const float* probs,
                                              const float* zs, float* scratch, const RowStats& st,
                                              float inv_t) {
  constexpr int W = THREADS / 64;
  float loss = 0.f;
  for (int e = threadIdx.x; e < a.K; e += THREADS) {
    const float p = probs[e];
    // p = 0 (too small for fp32, or no entry) adds 0; a NaN stays one
    if (p != 0.f) loss += p * (logf(p) - row_logprob(st, zs[e], inv_t));
  }
  loss = lanes_sum<64>(loss);
  if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = loss;
  __syncthreads();
  loss = 0.f;
  for (int w = 0; w < W; ++w) loss += scratch[w];
  __syncthreads();
  return loss;
}

// STATS: the row's statistics are taken here (else read); GRAD: its gradient
// is written.  parts > 1 with STATS: only the part's statistics are, into the
// workspace.
//
// Bound by memory.  4096 x 65536 bf16: the loss 97 us (5.5 TB/s), its gradient 228
// (4.7 TB/s read and written), both at once 270: a row's second read comes from
// the caches, which the rows that run at a time (three to a CU) fit.  Holding a row in
// registers between its two uses was slower: only one then fits a CU, and its
// loads stop while it writes.  515 x 30011 fp32: 16 and 25 us, 700 x 30011 17 and 38,
// both at once 44; these rows are too many to be cut and few enough to run all at the
// same time, two or three to a CU, so that none reads while they join their sums and
// the teacher's.
template <bool BF16, int THREADS, int U, bool STATS, bool GRAD>
__global__ __launch_bounds__(THREADS, 6) void distill_kernel(DistillArgs a, int parts) {
  using E = Elem<BF16>;
  constexpr int W = THREADS / 64;
  __shared__ float red[3 * W];
  __shared__ int cols[kMaxTeacher];
  __shared__ float probs[kMaxTeacher], zs[kMaxTeacher];
  const float inv_t = 1.f / a.r.temperature, k = kLog2e / a.r.temperature;
  const long long items = (long long)a.r.N * parts;
  for (long long it = blockIdx.x; it < items; it += gridDim.x) {
    const int row = (int)(it / parts), part = (int)(it - (long long)row * parts);
    const auto* z = static_cast<const typename E::T*>(a.r.z) + (long long)row * a.r.ld;
    Teacher<BF16, THREADS> teacher;
    float m, s;
    if (!STATS || parts == 1) teacher.fetch(a, row);
    if constexpr (STATS) {
      Found<W> none{nullptr, nullptr, nullptr, 0};
      Run<false> run = part_stats<BF16, THREADS, U, false, false>(z, a.r.V, part, parts, k, none);
      if (parts == 1) teacher.gather(a, z);
      run = run_block<THREADS>(run, k, red);
      m = run.m;
      s = run.s;
      if (parts > 1) {
        if (threadIdx.x == 0) run_store(static_cast<float*>(a.workspace) + 4 * it, run);
        continue;
      }
    } else {
      teacher.gather(a, z);
      m = a.stats[2LL * row];
      s = a.stats[2LL * row + 1];
    }
    const RowStats st = row_stats(m, s);
    PartGrad<BF16, THREADS, GRAD ? U : 1> pg(z, GRAD ? a.r.V : 0, part, parts);
    const float kept = teacher.probabilities(a, cols, probs, zs, red, k);
    if constexpr (STATS) {
      const float loss = distill_loss<THREADS>(a, probs, zs, red, st, inv_t);
      if (threadIdx.x == 0) {
        a.loss[row] = loss;
        a.stats[2LL * row] = m;
        a.stats[2LL * row + 1] = s;
      }
    }
    if constexpr (GRAD) {
      auto* dz = static_cast<typename E::T*>(a.dz) + (long long)row * a.ldd;
      // a row with no possible token, or no teacher, has no gradient
      const float g = s == 0.f || kept == 0.f ? 0.f : a.dloss[row] * inv_t;
      const float c0 = g == 0.f ? 0.f : g / s;
      for (int e = threadIdx.x; e < a.K; e += THREADS) {
        probs[e] = g == 0.f ? 0.f : -g * probs[e];
        if (g == 0.f) cols[e] = -1;
      }
      __syncthreads();  // (and the gathered logits are here: dz may be z)
      PointTerms<BF16, THREADS, kMaxTeacher, false> pt;
      pt.take(cols, probs, zs, a.K, z, a.r.V, part, parts, st.base, k, c0, 0.f);
      pg.template write<false>(dz, st.base, k, c0, 0.f);
      __syncthreads();
      pt.put(dz);
    }
    __syncthreads();
  }
}

// The parts of a row joined, and its loss; one workgroup per row.
template <bool BF16>
__global__ __launch_bounds__(256) void distill_join_kernel(DistillArgs a, int parts) {
  using E = Elem<BF16>;
  __shared__ float red[4];
  __shared__ int cols[kMaxTeacher];
  __shared__ float probs[kMaxTeacher], zs[kMaxTeacher];
  const float inv_t = 1.f / a.r.temperature, k = kLog2e / a.r.temperature;
  const float* ws = static_cast<const float*>(a.workspace);
  for (int row = blockIdx.x; row < a.r.N; row += gridDim.x) {
    const auto* z = static_cast<const typename E::T*>(a.r.z) + (long long)row * a.r.ld;
    const int lane = threadIdx.x & 63;
    Teacher<BF16, 256> teacher;
    teacher.fetch(a, row);
    Run<false> run;
    if (lane < parts) run = run_load<false>(ws + 4 * ((long long)row * parts + lane));
    teacher.gather(a, z);
    run_lanes<64>(run, k);
    const RowStats st = row_stats(run.m, run.s);
    teacher.probabilities(a, cols, probs, zs, red, k);
    const float loss = distill_loss<256>(a, probs, zs, red, st, inv_t);
    if (threadIdx.x == 0) {
      a.loss[row] = loss;
      a.stats[2LL * row] = run.m;
      a.stats[2LL * row + 1] = run.s;
    }
    __syncthreads();
  }
}

constexpr int kThreads = 512;
constexpr int kFewThreads = 256;
constexpr int kUnroll = 4;

// Parts a row is cut into where there are fewer rows than two to a CU.  Those of a
// gradient have at least a round of vectors; those of statistics, which another
// launch has to join, one for every load in flight, and a row of fewer than four
// such parts is left whole: the launch costs more than the rounds (us, cut and
// whole: 2 x 6637 bf16 6.7 and 5.3, 121 x 27584 9.3 and 7.1, its loss and gradient
// 17.9 and 15.9; with alternatives it is as much on the GPU, 14.0 and 18.2, as the
// launch takes from the host).
int parts_of(int N, int most) {
  const int want = (int)((511LL + N) / N), p = want < most ? want : most;
  return p < 1 ? 1 : p > kMaxParts ? kMaxParts : p;
}
int row_parts(int N, int V, bool bf16) {
  const int most = V / (kThreads * kUnroll * (bf16 ? 8 : 4));
  return most < 4 ? 1 : parts_of(N, most);
}
int grad_parts(int N, int V, bool bf16) {
  const int round = kThreads * (bf16 ? 8 : 4);
  return parts_of(N, V / round + (V % round != 0));
}
// Short rows that are not cut go to workgroups of 256 threads: what they wait for
// between loading and writing a row is a larger part then, and more rows at a
// time cover it.  16384 x 8192 bf16: forward 146 -> 72 us, gradient 161 -> 141;
// 8192 x 32000 bf16: forward 111 -> 98, gradient 205 -> 237 us.
bool short_rows(int V, bool bf16, int parts, bool grad_only) {
  return parts == 1 && V / (bf16 ? 8 : 4) <= (grad_only ? 2048 : 4096);
}

dim3 grid_of(long long items) { return dim3((unsigned)(items < kMaxGrid ? items : kMaxGrid)); }

template <bool BF16, bool TOP>
hipError_t logprob_run(const LogprobArgs& a, hipStream_t st) {
  const int parts = row_parts(a.r.N, a.r.V, BF16);
  const dim3 grid = grid_of((long long)a.r.N * parts);
  timing_before("logprobs", st);
  if (short_rows(a.r.V, BF16, parts, false))
    hipLaunchKernelGGL((logprob_kernel<BF16, kFewThreads, kUnroll, TOP>), grid, dim3(kFewThreads),
                       0, st, a, parts);
  else
    hipLaunchKernelGGL((logprob_kernel<BF16, kThreads, kUnroll, TOP>), grid, dim3(kThreads), 0, st,
                       a, parts);
  timing_after(st);
  if (hipError_t e = hipGetLastError()) return e;
  if (parts == 1) return hipSuccess;
  timing_before("logprobs_join", st);
  hipLaunchKernelGGL((logprob_join_kernel<BF16, TOP>), grid_of(a.r.N), dim3(256),
                     TOP ? sizeof(uint2) * parts * a.top : 0, st, a, parts);
  timing_after(st);
  return hipGetLastError();
}

template <bool BF16>
hipError_t logprob_grad_run(const LogprobGradArgs& a, hipStream_t st) {
  const int parts = grad_parts(a.r.N, a.r.V, BF16);
  const dim3 grid = grid_of((long long)a.r.N * parts);
  timing_before("logprobs_grad", st);
  if (short_rows(a.r.V, BF16, parts, true))
    hipLaunchKernelGGL((logprob_grad_kernel<BF16, kFewThreads, kUnroll>), grid, dim3(kFewThreads),
                       0, st, a, parts);
  else
    hipLaunchKernelGGL((logprob_grad_kernel<BF16, kThreads, kUnroll>), grid, dim3(kThreads), 0, st,
                       a, parts);
  timing_after(st);
  return hipGetLastError();
}

template <bool BF16, bool STATS, bool GRAD>
hipError_t distill_part(const DistillArgs& a, int parts, const char* label, hipStream_t st) {
  const dim3 grid = grid_of((long long)a.r.N * parts);
  timing_before(label, st);
  if (short_rows(a.r.V, BF16, parts, !STATS))
    hipLaunchKernelGGL((distill_kernel<BF16, kFewThreads, kUnroll, STATS, GRAD>), grid,
                       dim3(kFewThreads), 0, st, a, parts);
  else
    hipLaunchKernelGGL((distill_kernel<BF16, kThreads, kUnroll, STATS, GRAD>), grid,
                       dim3(kThreads), 0, st, a, parts);
  timing_after(st);
  return hipGetLastError();
}

template <bool BF16>
hipError_t distill_run(const DistillArgs& a, hipStream_t st) {
  const int parts = row_parts(a.r.N, a.r.V, BF16);
  if (a.loss) {
    if (a.dz && parts == 1) return distill_part<BF16, true, true>(a, 1, "distill", st);
    if (hipError_t e = distill_part<BF16, true, false>(a, parts, "distill", st)) return e;
    if (parts == 1) return hipSuccess;
    timing_before("distill_join", st);
    hipLaunchKernelGGL((distill_join_kernel<BF16>), grid_of(a.r.N), dim3(256), 0, st, a, parts);
    timing_after(st);
    if (hipError_t e = hipGetLastError()) return e;
  }
  if (!a.dz) return hipSuccess;
  return distill_part<BF16, false, true>(a, grad_parts(a.r.N, a.r.V, BF16), "distill_grad", st);
}

}  // namespace

size_t logprob_workspace_bytes(int N, int V, int bf16, int top) {
  const int parts = row_parts(N, V, bf16 != 0);
  return parts == 1 ? 0 : (size_t)N * parts * (16 + sizeof(uint2) * top);
}

hipError_t logprob_launch(const LogprobArgs& a, hipStream_t stream) {
  if (a.r.bf16)
    return a.top ? logprob_run<true, true>(a, stream) : logprob_run<true, false>(a, stream);
  return a.top ? logprob_run<false, true>(a, stream) : logprob_run<false, false>(a, stream);
}

hipError_t logprob_grad_launch(const LogprobGradArgs& a, hipStream_t stream) {
  return a.r.bf16 ? logprob_grad_run<true>(a, stream) : logprob_grad_run<false>(a, stream);
}

size_t distill_workspace_bytes(int N, int V, int bf16) {
  const int parts = row_parts(N, V, bf16 != 0);
  return parts == 1 ? 0 : (size_t)N * parts * 16;
}

hipError_t distill_launch(const DistillArgs& a, hipStream_t stream) {
  return a.r.bf16 ? distill_run<true>(a, stream) : distill_run<false>(a, stream);
}

}  // namespace sru
