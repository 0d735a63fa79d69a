// Gated linear recurrence of a channel j (every operation per channel):
//   s = sigma(r_t), g = sigma(i_t), k = c softplus(lam_j)
//   a_t = exp(-k s),  beta_t = sqrt(1 - a_t^2)
//   h_t = a_t h_{t-1} + beta_t g x_t
// A step that starts a new document has a = 0, beta = 1; a padded one leaves h
// as it is (a = 1, nothing added) and outputs 0.  The gradient, with G_t that
// of the loss by h_t and c_t = a_t G_t what step t hands to step t - 1:
//   G_t = dh_t + c_{t+1}
//   dx = G beta g,  di = G beta g x (1 - g),  dr = -k dla s (1 - s)
//   dla = G a (h_{t-1} - a g x / beta)           (of log a; beta depends on a)
//   dlam = -c sigma(lam) sum_t dla s,  dh0 = c_0
//
// A step is an affine map of the state, h -> A h + B, and so is any run of
// steps; both directions are one scan over such maps.  A wave holds some
// steps (kLruForward or kLruSteps) of 64 lanes, VEC channels each, in registers,
// a workgroup up to kLruWaves
// waves, consecutive in time: a segment.  Maps are joined in the workgroup
// through LDS and, where a sequence has several segments, across workgroups
// through one 64-bit word per channel and segment: everything is read once.
//
// A map with A = 0 forgets what came before: that is how a new document's
// start, and a state that is known, are written (a state of NaN before a new
// document must not reach it through 0 * NaN).  Products of decays that are
// merely small stay above 0.
#include <algorithm>

#include "sru_device.h"
#include "sru_lm.h"

namespace sru {
namespace {

constexpr int T = kLruSteps;
constexpr int kLook = 8;   // segments of a block
constexpr int kFewChannels = 4096;
constexpr float kTiny = 1.17549435e-38f;
constexpr float kLog2e = 1.44269504088896341f;

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }

struct Map {
  float A, B;
};
__device__ __forceinline__ float apply(Map m, float h) { return m.A == 0.f ? m.B : fmaf(m.A, h, m.B); }
// `late` after `early`
__device__ __forceinline__ Map join(Map late, Map early) {
  if (late.A == 0.f) return late;
  return Map{early.A == 0.f ? 0.f : fmaxf(late.A * early.A, kTiny), fmaf(late.A, early.B, late.B)};
}

// Keeps a value in a register from here on: left alone, the compiler moves its
// last operations to where it is used and carries their operands instead.
__device__ __forceinline__ void hold(float& x) { asm volatile("" : "+v"(x)); }

// VEC consecutive values of an activation type, loaded whole and kept packed
// (bf16 pairs in one register) until they are used.
template <bool BF16, int VEC>
struct Pack;
template <>
struct Pack<true, 1> {
  uint16_t u;
  __device__ __forceinline__ float get(int) const { return __uint_as_float((unsigned)u << 16); }
  __device__ __forceinline__ void put(const float (&f)[1]) {
    u = __builtin_bit_cast(uint16_t, (__bf16)f[0]);
  }
};
template <>
struct Pack<true, 2> {
  unsigned u;
  __device__ __forceinline__ float get(int v) const {
    return __uint_as_float(v ? u & 0xffff0000u : u << 16);
  }
  __device__ __forceinline__ void put(const float (&f)[2]) {
    u = (unsigned)__builtin_bit_cast(uint16_t, (__bf16)f[0]) |
        ((unsigned)__builtin_bit_cast(uint16_t, (__bf16)f[1]) << 16);
  }
};
template <>
struct Pack<false, 1> {
  float u;
  __device__ __forceinline__ float get(int) const { return u; }
  __device__ __forceinline__ void put(const float (&f)[1]) { u = f[0]; }
};
template <>
struct Pack<false, 2> {
  float2 u;
  __device__ __forceinline__ float get(int v) const { return v ? u.y : u.x; }
  __device__ __forceinline__ void put(const float (&f)[2]) { u = make_float2(f[0], f[1]); }
};

// Where a wave's and its lanes' channels lie: a workgroup's lanes are 64 VEC
// features of one sequence, so that what depends on the sequence and the step
// alone (addresses, padding, new documents) is worked out once for the wave.
struct Lane {
  int b;            // sequence, the same for the workgroup
  int j;            // the lane's first feature
  bool live;        // j < d
  long long chan;   // b * d + j
};
template <int VEC>
__device__ __forceinline__ Lane lane_of(const LruArgs& a, int group) {
  const int per = (a.d + 64 * VEC - 1) / (64 * VEC);
  Lane n;
  n.b = group / per;
  n.j = (group - n.b * per) * 64 * VEC + (threadIdx.x & 63) * VEC;
  n.live = n.j < a.d;
  n.chan = (long long)n.b * a.d + n.j;
  return n;
}

// A tensor at a wave's steps: the wave's address, and the lane's offset in it.
template <bool BF16, int VEC>
struct Ptr {
  using P = Pack<BF16, VEC>;
  char* p;
  long long step;  // bytes
  unsigned off;
  __device__ __forceinline__ Ptr(const Seq& s, const Lane& n, int t0) {
    constexpr int ES = BF16 ? 2 : 4;
    step = ES * s.st;
    p = static_cast<char*>(const_cast<void*>(s.p)) + t0 * step + ES * (n.b * s.sb);
    off = ES * (unsigned)n.j;
  }
  __device__ __forceinline__ P load(int u) const {
    return *reinterpret_cast<const P*>(p + u * step + off);
  }
  __device__ __forceinline__ void store(int u, const float (&f)[VEC]) const {
    P o;
    o.put(f);
    *reinterpret_cast<P*>(p + u * step + off) = o;
  }
};

// A tensor's packed values at a wave's N steps from t0, zeros where there are none.
template <bool BF16, int VEC, int N>
__device__ __forceinline__ void load_steps(const LruArgs& a, const Seq& s, const Lane& n, int t0,
                                           Pack<BF16, VEC> (&x)[N]) {
  const Ptr<BF16, VEC> p(s, n, t0);
#pragma unroll
  for (int u = 0; u < N; ++u) x[u] = Pack<BF16, VEC>{};
  if (!n.live) return;
  if (t0 + N <= a.L) {
#pragma unroll
    for (int u = 0; u < N; ++u) x[u] = p.load(u);
  } else {
#pragma unroll
    for (int u = 0; u < N; ++u)
      if (t0 + u < a.L) x[u] = p.load(u);
  }
}

// What a wave knows of its N steps: how many there are, and bit u of pad, fresh
// for step u.  Lane u reads step u's marks.
struct Flags {
  int count;
  unsigned pad, fresh;
};
template <bool FLAGS, int N>
__device__ __forceinline__ Flags flags_of(const LruArgs& a, const Lane& n, int t0) {
  Flags f{min(max(a.L - t0, 0), N), 0, 0};
  if constexpr (FLAGS) {
    const int u = threadIdx.x & 63;
    const long long o = (long long)(t0 + u) * a.B + n.b;
    if (a.mask) f.pad = (unsigned)__ballot(u < f.count && a.mask[o] != 0);
    if (a.reset) f.fresh = (unsigned)__ballot(u < f.count && a.reset[o] != 0) & ~f.pad;
  }
  return f;
}

// A step's decay a = e^-y and q = 1 - a^2 from y = k s.  Both come from w = 1 -
// a, by the series of 1 - e^-y where that would cancel (its next term is y^5 /
// 720, below 2^-25 of w here): q = w (2 - w), and a = 1 - w is rounded once, to
// nearest.  A state carried on over a thousand steps multiplies as many decays
// near 1: the error of the hardware's 2^x there, which leans to one side, would
// add up.
// SERIES: every y of the wave is below kSeriesEnd, and the step keeps w; else it
// keeps y.
constexpr float kSeriesEnd = 0.11f;
struct Decay {
  float a, q;
};
__device__ __forceinline__ float series(float y) {
  float p = fmaf(y, 1.f / 120.f, -1.f / 24.f);
  p = fmaf(y, p, 1.f / 6.f);
  p = fmaf(y, p, -0.5f);
  return fmaf(y, p, 1.f) * y;
}
template <bool SERIES>
__device__ __forceinline__ float decay_kept(float k, float s) {
  return SERIES ? series(k * s) : k * s;
}
template <bool SERIES>
__device__ __forceinline__ Decay decay_of(float kept) {
  if constexpr (SERIES) return Decay{1.f - kept, kept * (2.f - kept)};
  const float p = series(kept), e = fmaxf(exp2_hw(-kLog2e * kept), kTiny);
  const bool small = kept < kSeriesEnd;
  const float w = small ? p : 1.f - e;
  return Decay{small ? 1.f - p : e, w * (2.f - w)};
}

// k = c softplus(lam) of a feature
__device__ __forceinline__ float decay_rate(const LruArgs& a, int j) {
  const float l = a.lam[j];
  return a.c * (fmaxf(l, 0.f) + log1pf(expf(-fabsf(l))));
}
// k of the lane's channels.  With several segments the call's first kernel has
// worked them out; else the first wave does, for all.  Returns whether all of
// the wave's series converge (s <= 1).
template <int VEC>
__device__ __forceinline__ bool decay_rates(const LruArgs& a, const float* rates, const Lane& n,
                                            float* lds, float (&k)[VEC]) {
  if (rates) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) k[v] = n.live ? rates[n.j + v] : 0.f;
  } else {
    if (threadIdx.x < 64) {
#pragma unroll
      for (int v = 0; v < VEC; ++v)
        lds[v * 64 + threadIdx.x] = n.live ? decay_rate(a, n.j + v) : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < VEC; ++v) k[v] = lds[v * 64 + (threadIdx.x & 63)];
  }
  bool beyond = false;
#pragma unroll
  for (int v = 0; v < VEC; ++v) beyond |= !(k[v] < kSeriesEnd);
  return !__any(beyond);
}

// ------------------------------------------------------ maps across segments
// One word per channel and segment: a map (A in the upper half), all ones
// while there is none.  A is never NaN, so no map looks like that.
constexpr unsigned long long kEmpty = ~0ull;
__device__ __forceinline__ unsigned long long word_of(Map m) {
  return ((unsigned long long)__float_as_uint(m.A) << 32) | __float_as_uint(m.B);
}
__device__ __forceinline__ Map map_of(unsigned long long w) {
  return Map{__uint_as_float((unsigned)(w >> 32)), __uint_as_float((unsigned)w)};
}

struct Chain {
  unsigned* tickets;          // one a lane group, kTicketPitch apart
  unsigned long long* words;  // [nseg, B * d]
  float* rates;               // [d]; nullptr with one segment
  int nseg, groups;
};
constexpr int kTicketPitch = 16;  // a cache line each: all start at the same time

// The segment (in the order of the scan) that a workgroup of a lane group takes:
// tickets are handed out as workgroups start, and a segment only waits for
// those with lower tickets.  These have started, so they get on whatever else
// waits: every wait ends.
__device__ __forceinline__ int take_ticket(const Chain& c, int group, unsigned* lds) {
  if (c.nseg == 1) return 0;
  if (threadIdx.x == 0)
    *lds = __hip_atomic_fetch_add(c.tickets + (long long)group * kTicketPitch, 1u,
                                  __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  return __builtin_amdgcn_readfirstlane(*lds);
}

template <int VEC>
__device__ __forceinline__ void publish(const Chain& c, const LruArgs& a, const Lane& n, int rank,
                                        const Map (&m)[VEC]) {
  if (!n.live) return;
  unsigned long long* w = c.words + (long long)rank * a.B * a.d + n.chan;
#pragma unroll
  for (int v = 0; v < VEC; ++v)
    __hip_atomic_store(w + v, word_of(m[v]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The map in a word once it is there.  The wait ends by the order of the tickets;
// its bound (seconds) keeps a mistake there from hanging the GPU: NaN then.
__device__ __forceinline__ Map wait_for(const unsigned long long* word, bool live) {
  unsigned long long x = kEmpty;
#pragma unroll 1
  for (int spin = 0; live && spin < (1 << 22); ++spin) {
    x = __hip_atomic_load(word, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (x != kEmpty) break;
    __builtin_amdgcn_s_sleep(1);
  }
  return map_of(x);
}

// The maps of a workgroup's waves, in LDS in the order of the scan (`place` of
// a wave's steps in it), joined: the state that enters the wave's steps, and
// the segment's map where the state entering that is not known yet.
template <int U, int VEC>
__device__ __forceinline__ void enter_wave(const Map* maps, int place, const float (&seg_in)[VEC],
                                           float (&in)[VEC]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int v = 0; v < VEC; ++v) in[v] = seg_in[v];
#pragma unroll U
  for (int w = 0; w < place; ++w)
#pragma unroll
    for (int v = 0; v < VEC; ++v) in[v] = apply(maps[(w * VEC + v) * 64 + lane], in[v]);
}

// The state that enters the segment; `first` is what enters rank 0.  Segments
// come in blocks of kLook.  The last one of a block leaves the state after the
// block (a map with A = 0) in its word, the others their own map; a segment
// takes the state before its block and the maps of its block before it.  All
// are joined in the order of the scan, the state last of all, so that a state
// passes a block in one hop of a word, and the result does not depend on which
// workgroup ran when.  win: kLook * 64 * VEC maps.
// U: how far the loops over maps are unrolled (their reads take registers).
template <int U, int VEC>
__device__ __forceinline__ void join_segments(const Chain& c, const LruArgs& a, const Lane& n,
                                              int rank, int waves, const Map* maps, Map* win,
                                              const float (&first)[VEC], float (&seg_in)[VEC]) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int v = 0; v < VEC; ++v) seg_in[v] = first[v];
  if (c.nseg == 1) return;
  const int inside = rank % kLook, block = rank - inside;
  const bool mine = wave == 0 && rank + 1 < c.nseg, leaves = inside == kLook - 1;
  const long long lanes = (long long)a.B * a.d;
  unsigned long long* const words = c.words + n.chan;
  Map seg[VEC];
  if (mine) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) seg[v] = maps[v * 64 + lane];
#pragma unroll U
    for (int w = 1; w < waves; ++w)
#pragma unroll
      for (int v = 0; v < VEC; ++v) seg[v] = join(maps[(w * VEC + v) * 64 + lane], seg[v]);
    if (!leaves) publish<VEC>(c, a, n, rank, seg);
  }
  if (rank == 0) return;
#pragma unroll 1
  for (int e = wave; e < inside; e += waves) {
#pragma unroll
    for (int v = 0; v < VEC; ++v)
      win[(e * VEC + v) * 64 + lane] = wait_for(words + (block + e) * lanes + v, n.live);
  }
  __syncthreads();
  if (mine && leaves) {
    // the whole block as one map, before the state is there
    Map all[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) all[v] = win[v * 64 + lane];
#pragma unroll U
    for (int e = 1; e < inside; ++e)
#pragma unroll
      for (int v = 0; v < VEC; ++v) all[v] = join(win[(e * VEC + v) * 64 + lane], all[v]);
#pragma unroll
    for (int v = 0; v < VEC; ++v) seg[v] = join(seg[v], all[v]);
  }
  if (block > 0) {
#pragma unroll
    for (int v = 0; v < VEC; ++v)
      seg_in[v] = wait_for(words + (block - 1) * lanes + v, n.live).B;
  }
  if (mine && leaves) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) seg[v] = Map{0.f, apply(seg[v], seg_in[v])};
    publish<VEC>(c, a, n, rank, seg);
  }
#pragma unroll U
  for (int e = 0; e < inside; ++e)
#pragma unroll
    for (int v = 0; v < VEC; ++v) seg_in[v] = apply(win[(e * VEC + v) * 64 + lane], seg_in[v]);
}

// Empties the words (two at a time) and the tickets and works out the rates.
__global__ __launch_bounds__(256) void lru_clear_kernel(LruArgs a, Chain c, long long pairs) {
  const long long step = (long long)gridDim.x * 256;
  const long long first = (long long)blockIdx.x * 256 + threadIdx.x;
  ulonglong2* w = reinterpret_cast<ulonglong2*>(c.words);
  for (long long i = first; i < pairs; i += step) w[i] = make_ulonglong2(kEmpty, kEmpty);
  for (long long i = first; i < (long long)c.groups * kTicketPitch; i += step) c.tickets[i] = 0;
  for (long long i = first; i < a.d; i += step) c.rates[i] = decay_rate(a, (int)i);
}

// -------------------------------------------------------------------- forward
// A wave's steps as maps h -> A h + B (A of a document's first step is 0), and
// the map of them all.  FLAGS: some step may be missing, be padded or start a
// document.
template <bool FLAGS, bool SERIES, bool BF16, int VEC, int N>
__device__ __forceinline__ void step_maps(const Pack<BF16, VEC> (&x)[N],
                                          const Pack<BF16, VEC> (&r)[N],
                                          const Pack<BF16, VEC> (&i)[N], const float (&k)[VEC],
                                          const Flags& f, float (&A)[N][VEC], float (&Bv)[N][VEC],
                                          Map (&all)[VEC]) {
#pragma unroll
  for (int v = 0; v < VEC; ++v) all[v] = Map{1.f, 0.f};
#pragma unroll
  for (int u = 0; u < N; ++u) {
    if (FLAGS && u >= f.count) continue;
    const bool pad = FLAGS && (f.pad >> u & 1), fresh = FLAGS && (f.fresh >> u & 1);
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      const float s = sigmoid_fast(r[u].get(v)), g = sigmoid_fast(i[u].get(v));
      const Decay dc = decay_of<SERIES>(decay_kept<SERIES>(k[v], s));
      const float gx = g * x[u].get(v);
      A[u][v] = pad ? 1.f : fresh ? 0.f : dc.a;
      Bv[u][v] = pad ? 0.f : fresh ? gx : __builtin_amdgcn_sqrtf(dc.q) * gx;
      all[v].B = fresh ? gx : fmaf(A[u][v], all[v].B, Bv[u][v]);
      all[v].A *= A[u][v];
    }
  }
  const bool anew = FLAGS && f.fresh != 0;
#pragma unroll
  for (int v = 0; v < VEC; ++v) all[v].A = anew ? 0.f : fmaxf(all[v].A, kTiny);
}

// The outputs of the steps once the state entering them is known.
template <bool FLAGS, bool BF16, int VEC, int N>
__device__ __forceinline__ void run_steps(const LruArgs& a, const Lane& n, int t0, const Flags& f,
                                          const float (&A)[N][VEC], const float (&Bv)[N][VEC],
                                          float (&h)[VEC]) {
  const Ptr<BF16, VEC> out(a.h, n, t0);
  float* kept = a.states ? a.states + (long long)(t0 / T) * a.B * a.d + n.chan : nullptr;
#pragma unroll
  for (int u = 0; u < N; ++u) {
    if (FLAGS && u >= f.count) continue;
    const bool pad = FLAGS && (f.pad >> u & 1), fresh = FLAGS && (f.fresh >> u & 1);
    if (u % T == 0 && kept) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) kept[(long long)(u / T) * a.B * a.d + v] = h[v];
    }
    float y[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      h[v] = fresh ? Bv[u][v] : fmaf(A[u][v], h[v], Bv[u][v]);
      y[v] = pad ? 0.f : h[v];
    }
    out.store(u, y);
  }
}

// A workgroup's place in the scan.
struct Place {
  int rank, waves, wave, t0;
};

template <bool FLAGS, bool SERIES, bool BF16, int VEC, int N>
__device__ __forceinline__ void lru_body(const LruArgs& a, const Chain& c, const Lane& n,
                                         const Place& p, const Flags& f, const float (&k)[VEC],
                                         const float (&first)[VEC], const Pack<BF16, VEC> (&x)[N],
                                         const Pack<BF16, VEC> (&r)[N],
                                         const Pack<BF16, VEC> (&i)[N], Map* maps, Map* win) {
  float A[N][VEC], Bv[N][VEC], seg_in[VEC], h[VEC];
  Map m[VEC];
  step_maps<FLAGS, SERIES, BF16, VEC, N>(x, r, i, k, f, A, Bv, m);
#pragma unroll
  for (int v = 0; v < VEC; ++v) maps[(p.wave * VEC + v) * 64 + (threadIdx.x & 63)] = m[v];
  __syncthreads();
  join_segments<4>(c, a, n, p.rank, p.waves, maps, win, first, seg_in);
  enter_wave<4>(maps, p.wave, seg_in, h);
  if (!n.live || f.count == 0) return;
  run_steps<FLAGS, BF16, VEC, N>(a, n, p.t0, f, A, Bv, h);
  if (a.h_last && p.t0 + N >= a.L) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) a.h_last[n.chan + v] = h[v];
  }
}

// FLAGS: there is padding or a new document somewhere, or a wave's last steps
// are missing.  All waves of a workgroup have the same channels, so all take
// the same body.
template <bool BF16, int VEC, bool FLAGS, int W>
__global__ __launch_bounds__(64 * W, W == 16 ? 4 : 5) void lru_kernel(LruArgs a, Chain c) {
  constexpr int N = kLruForward;
  __shared__ Map maps[W * VEC * 64], win[kLook * VEC * 64];
  __shared__ float rates[VEC * 64];
  __shared__ unsigned ticket;
  const int group = blockIdx.x % (unsigned)c.groups;
  Place p;
  p.rank = take_ticket(c, group, &ticket);
  p.waves = blockDim.x >> 6;
  p.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  p.t0 = (p.rank * p.waves + p.wave) * N;
  const Lane n = lane_of<VEC>(a, group);

  Pack<BF16, VEC> x[N], r[N], i[N];
  load_steps<BF16, VEC, N>(a, a.r, n, p.t0, r);
  load_steps<BF16, VEC, N>(a, a.i, n, p.t0, i);
  load_steps<BF16, VEC, N>(a, a.x, n, p.t0, x);
  const Flags f = flags_of<FLAGS, N>(a, n, p.t0);
  float k[VEC], first[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) first[v] = a.h0 && n.live ? a.h0[n.chan + v] : 0.f;
  if (decay_rates<VEC>(a, c.rates, n, rates, k))
    lru_body<FLAGS, true, BF16, VEC, N>(a, c, n, p, f, k, first, x, r, i, maps, win);
  else
    lru_body<FLAGS, false, BF16, VEC, N>(a, c, n, p, f, k, first, x, r, i, maps, win);
}

// ------------------------------------------------------------------- gradient
// What a wave's steps need once the gradient entering them is known, per step:
//   A = a, e = beta g, E = s (h_{t-1} - a g x / beta), P = k (s - 1), X = x (1 - g)
// so that with G = dh + c:  dx = G e, di = dx X, dla s = G A E, dr = (dla s) P.
// The states go along (h enters), and so does the map of the gradient c that the
// steps hand on, c_t = a_t (c_{t+1} + dh_t): taken in this order it is
//   A = prod a,  B = sum_u (prod_{v <= u} a_v) dh_u.
template <int VEC>
struct GradSteps {
  float A[T][VEC], e[T][VEC], E[T][VEC], P[T][VEC], X[T][VEC];
};
template <bool FLAGS, bool SERIES, bool BF16, int VEC>
__device__ __forceinline__ void grad_maps(const Pack<BF16, VEC> (&x)[T],
                                          const Pack<BF16, VEC> (&r)[T],
                                          const Pack<BF16, VEC> (&i)[T],
                                          const Pack<BF16, VEC> (&dh)[T], const float (&k)[VEC],
                                          const Flags& f, float (&h)[VEC], GradSteps<VEC>& st,
                                          Map (&all)[VEC]) {
#pragma unroll
  for (int v = 0; v < VEC; ++v) all[v] = Map{1.f, 0.f};
#pragma unroll
  for (int u = 0; u < T; ++u) {
    const bool pad = FLAGS && ((f.pad >> u & 1) || u >= f.count);
    const bool fresh = FLAGS && (f.fresh >> u & 1);
    // a document starts here or did before: nothing later is handed on
    const bool cut = FLAGS && (f.fresh & (2u << u) - 1) != 0;
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      const float s = sigmoid_fast(r[u].get(v)), g = sigmoid_fast(i[u].get(v));
      const Decay dc = decay_of<SERIES>(decay_kept<SERIES>(k[v], s));
      // a decay of 1 (no rate, or a gate that is shut) adds nothing, and its
      // root's slope, which has no bound, meets a rate of 0: keep it finite
      const float q = fmaxf(dc.q, kTiny);
      const float rb = __builtin_amdgcn_rsqf(q);  // 1 / beta
      const float xv = x[u].get(v), gx = g * xv;
      const float e = fresh ? g : q * rb * g;
      st.A[u][v] = dc.a;
      st.e[u][v] = e;
      st.E[u][v] = s * fmaf(-(dc.a * rb), gx, h[v]);
      st.P[u][v] = fmaf(k[v], s, -k[v]);
      st.X[u][v] = xv - gx;
      const float hn = fresh ? gx : fmaf(dc.a, h[v], e * xv);
      h[v] = pad ? h[v] : hn;
      const float A = all[v].A * dc.a;
      const float B = fmaf(A, dh[u].get(v), all[v].B);
      all[v].A = pad ? all[v].A : A;
      all[v].B = pad || cut ? all[v].B : B;
      hold(st.A[u][v]), hold(st.e[u][v]), hold(st.E[u][v]), hold(st.P[u][v]), hold(st.X[u][v]);
    }
  }
  const bool anew = FLAGS && f.fresh != 0;
#pragma unroll
  for (int v = 0; v < VEC; ++v) all[v].A = anew ? 0.f : fmaxf(all[v].A, kTiny);
}

// The gradients of a wave's steps; leaves carry as it is handed on, and -sum dla
// s in acc.
template <bool FLAGS, bool BF16, int VEC>
__device__ __forceinline__ void grad_steps(const LruArgs& a, const Lane& n, int t0,
                                           const Pack<BF16, VEC> (&dh)[T],
                                           const GradSteps<VEC>& st, const Flags& f,
                                           float (&carry)[VEC], float (&acc)[VEC]) {
  const Ptr<BF16, VEC> pdx(a.dx, n, t0), pdr(a.dr, n, t0), pdi(a.di, n, t0);
#pragma unroll
  for (int u = T - 1; u >= 0; --u) {
    if (FLAGS && u >= f.count) continue;
    const bool pad = FLAGS && (f.pad >> u & 1), fresh = FLAGS && (f.fresh >> u & 1);
    float dx[VEC], dr[VEC], di[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      const float G = dh[u].get(v) + carry[v];
      // a new document's start depends on no decay and hands nothing on
      const float ga = fresh ? 0.f : G * st.A[u][v];
      const float dls = pad || fresh ? 0.f : ga * st.E[u][v];
      acc[v] -= dls;
      const float ge = G * st.e[u][v];
      dx[v] = pad ? 0.f : ge;
      dr[v] = pad || fresh ? 0.f : dls * st.P[u][v];
      di[v] = pad ? 0.f : ge * st.X[u][v];
      carry[v] = pad ? carry[v] : ga;
    }
    pdx.store(u, dx);
    pdr.store(u, dr);
    pdi.store(u, di);
  }
}

template <bool FLAGS, bool SERIES, bool BF16, int VEC>
__device__ __forceinline__ void grad_body(const LruArgs& a, const Chain& c, const Lane& n,
                                          const Place& p, const Flags& f, const float (&k)[VEC],
                                          const float (&first)[VEC], float (&h)[VEC],
                                          const Pack<BF16, VEC> (&x)[T],
                                          const Pack<BF16, VEC> (&r)[T],
                                          const Pack<BF16, VEC> (&i)[T],
                                          const Pack<BF16, VEC> (&dh)[T], Map* maps, Map* win,
                                          float (&acc)[VEC]) {
  GradSteps<VEC> st;
  float seg_in[VEC], carry[VEC];
  Map m[VEC];
  grad_maps<FLAGS, SERIES, BF16, VEC>(x, r, i, dh, k, f, h, st, m);
  const int place = p.waves - 1 - p.wave;
#pragma unroll
  for (int v = 0; v < VEC; ++v)
    maps[(place * VEC + v) * 64 + (threadIdx.x & 63)] = f.count ? m[v] : Map{1.f, 0.f};
  __syncthreads();
  join_segments<1>(c, a, n, p.rank, p.waves, maps, win, first, seg_in);
  enter_wave<1>(maps, place, seg_in, carry);
  if (!n.live || f.count == 0) return;
  grad_steps<FLAGS, BF16, VEC>(a, n, p.t0, dh, st, f, carry, acc);
  if (a.dh0 && p.t0 == 0) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) a.dh0[n.chan + v] = carry[v];
  }
}

// The scan runs from the last step to the first: rank 0 is the last segment,
// and a workgroup's last wave comes first.  sums: [nseg, B, d] of -sum dla s.
template <bool BF16, int VEC, bool FLAGS, int W>
__global__ __launch_bounds__(64 * W, 3) void lru_grad_kernel(LruArgs a, Chain c, float* sums) {
  __shared__ Map maps[W * VEC * 64], win[kLook * VEC * 64];
  __shared__ float rates[VEC * 64];
  __shared__ unsigned ticket;
  const int group = blockIdx.x % (unsigned)c.groups;
  Place p;
  p.rank = take_ticket(c, group, &ticket);
  p.waves = blockDim.x >> 6;
  p.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int seg = c.nseg - 1 - p.rank;
  p.t0 = (seg * p.waves + p.wave) * T;
  const Lane n = lane_of<VEC>(a, group);

  Pack<BF16, VEC> x[T], r[T], i[T], dh[T];
  load_steps<BF16, VEC, T>(a, a.r, n, p.t0, r);
  load_steps<BF16, VEC, T>(a, a.dh, n, p.t0, dh);
  load_steps<BF16, VEC, T>(a, a.i, n, p.t0, i);
  load_steps<BF16, VEC, T>(a, a.x, n, p.t0, x);
  const Flags f = flags_of<FLAGS, T>(a, n, p.t0);
  float k[VEC], first[VEC], h[VEC], acc[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    first[v] = a.dh_last && n.live ? a.dh_last[n.chan + v] : 0.f;
    h[v] = n.live && f.count ? a.states[(long long)(p.t0 / T) * a.B * a.d + n.chan + v] : 0.f;
    acc[v] = 0.f;
  }
  if (decay_rates<VEC>(a, c.rates, n, rates, k))
    grad_body<FLAGS, true, BF16, VEC>(a, c, n, p, f, k, first, h, x, r, i, dh, maps, win, acc);
  else
    grad_body<FLAGS, false, BF16, VEC>(a, c, n, p, f, k, first, h, x, r, i, dh, maps, win, acc);

  // the waves' sums in a fixed order
  float* red = reinterpret_cast<float*>(win);
  const int lane = threadIdx.x & 63;
  __syncthreads();
#pragma unroll
  for (int v = 0; v < VEC; ++v) red[(p.wave * VEC + v) * 64 + lane] = acc[v];
  __syncthreads();
  if (p.wave == 0 && n.live) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      float t = acc[v];
      for (int q = 1; q < p.waves; ++q) t += red[(q * VEC + v) * 64 + lane];
      sums[(long long)seg * a.B * a.d + n.chan + v] = t;
    }
  }
}

// dlam = c sigma(lam) sum over rows of [rows, d]: 64 features a workgroup, its
// 16 waves take every 16th row and meet in a fixed order.
__global__ __launch_bounds__(1024) void lru_sums_kernel(LruArgs a, const float* sums,
                                                        long long rows) {
  __shared__ float red[16 * 64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int j = blockIdx.x * 64 + lane;
  float s = 0.f;
  if (j < a.d) {
#pragma unroll 8
    for (long long row = w; row < rows; row += 16) s += sums[row * a.d + j];
  }
  red[w * 64 + lane] = s;
  __syncthreads();
  if (w == 0 && j < a.d) {
#pragma unroll
    for (int i = 1; i < 16; ++i) s += red[i * 64 + lane];
    a.dlam[j] = a.c * s / (1.f + expf(-a.lam[j]));
  }
}

// Waves of a workgroup and segments of a sequence.  Small workgroups overlap
// their loads with each other's arithmetic best; few channels make many segments
// in a row, where what counts is how many hops a state takes: larger ones.
int steps_of(bool grad) { return grad ? T : kLruForward; }
struct Plan {
  int full, waves, nseg;
};
Plan plan(int L, int B, int d, bool grad) {
  const int n = (L + steps_of(grad) - 1) / steps_of(grad);
  const bool few = (long long)B * d < kFewChannels;
  Plan p;
  p.full = grad ? (few ? 12 : 4) : (few ? 16 : 8);
  p.waves = std::min(n, p.full);
  p.nseg = (n + p.full - 1) / p.full;
  return p;
}

// Two channels a lane where every pair of features lies on its own size.
template <typename F>
bool pairs_ok(const LruArgs& a, F each) {
  if (a.d & 1) return false;
  const uintptr_t pair = a.bf16 ? 3 : 7;
  bool ok = true;
  each([&](const Seq& s) {
    ok = ok && ((reinterpret_cast<uintptr_t>(s.p) & pair) == 0) && !(s.st & 1) && !(s.sb & 1);
  });
  return ok;
}

size_t align_up(size_t x) { return (x + 255) / 256 * 256; }
// Workspace of several segments: words (an even number), tickets (of as many
// workgroups as one channel a lane makes), rates.
struct Layout {
  size_t words, tickets, rates, total;
};
Layout layout(int L, int B, int d, bool grad) {
  const int nseg = plan(L, B, d, grad).nseg;
  const size_t lanes = (size_t)B * d, groups = (size_t)B * ((d + 63) / 64);
  Layout l;
  l.words = sizeof(unsigned long long) * ((nseg * lanes + 1) / 2 * 2);
  l.tickets = align_up(l.words);
  l.rates = l.tickets + align_up(sizeof(unsigned) * kTicketPitch * groups);
  l.total = nseg == 1 ? 0 : l.rates + align_up(sizeof(float) * d);
  return l;
}

hipError_t clear(const Chain& c, const LruArgs& a, hipStream_t st) {
  const long long pairs = ((long long)c.nseg * a.B * a.d + 1) / 2;
  const long long most = std::max({pairs, (long long)c.groups * kTicketPitch, (long long)a.d});
  const long long blocks = (most + 511) / 512;
  timing_before("lru_clear", st);
  hipLaunchKernelGGL(lru_clear_kernel, dim3((unsigned)std::min(blocks, 2048LL)), dim3(256), 0, st,
                     a, c, pairs);
  timing_after(st);
  return hipGetLastError();
}

template <bool BF16, int VEC, bool FLAGS>
void launch(const LruArgs& a, const Chain& c, const Plan& p, float* sums, bool grad,
            hipStream_t st) {
  const dim3 grid((unsigned)c.groups * p.nseg), block(64 * p.waves);
  if (grad && p.full == 4)
    hipLaunchKernelGGL((lru_grad_kernel<BF16, VEC, FLAGS, 4>), grid, block, 0, st, a, c, sums);
  else if (grad)
    hipLaunchKernelGGL((lru_grad_kernel<BF16, VEC, FLAGS, 12>), grid, block, 0, st, a, c, sums);
  else if (p.full == 8)
    hipLaunchKernelGGL((lru_kernel<BF16, VEC, FLAGS, 8>), grid, block, 0, st, a, c);
  else
    hipLaunchKernelGGL((lru_kernel<BF16, VEC, FLAGS, 16>), grid, block, 0, st, a, c);
}

template <bool BF16, int VEC>
hipError_t run(const LruArgs& a, bool grad, hipStream_t st) {
  const Plan p = plan(a.L, a.B, a.d, grad);
  Chain c{};
  c.nseg = p.nseg;
  c.groups = a.B * ((a.d + 64 * VEC - 1) / (64 * VEC));
  char* ws = static_cast<char*>(a.workspace);
  const Layout l = layout(a.L, a.B, a.d, grad);
  if (p.nseg > 1) {
    c.words = reinterpret_cast<unsigned long long*>(ws);
    c.tickets = reinterpret_cast<unsigned*>(ws + l.tickets);
    c.rates = reinterpret_cast<float*>(ws + l.rates);
    if (hipError_t e = clear(c, a, st)) return e;
  }
  float* sums = reinterpret_cast<float*>(ws + l.total);
  timing_before(grad ? "lru_grad" : "lru", st);
  if (a.mask || a.reset || a.L % steps_of(grad))
    launch<BF16, VEC, true>(a, c, p, sums, grad, st);
  else
    launch<BF16, VEC, false>(a, c, p, sums, grad, st);
  timing_after(st);
  if (hipError_t e = hipGetLastError()) return e;
  if (!grad) return hipSuccess;
  timing_before("lru_sums", st);
  hipLaunchKernelGGL(lru_sums_kernel, dim3((a.d + 63) / 64), dim3(1024), 0, st, a, sums,
                     (long long)p.nseg * a.B);
  timing_after(st);
  return hipGetLastError();
}

hipError_t dispatch(const LruArgs& a, bool grad, bool pairs, hipStream_t st) {
  if (a.bf16) return pairs ? run<true, 2>(a, grad, st) : run<true, 1>(a, grad, st);
  return pairs && !grad ? run<false, 2>(a, grad, st) : run<false, 1>(a, grad, st);
}

}  // namespace

size_t lru_workspace_bytes(int L, int B, int d) { return layout(L, B, d, false).total; }

size_t lru_grad_workspace_bytes(int L, int B, int d) {
  return layout(L, B, d, true).total + sizeof(float) * (size_t)plan(L, B, d, true).nseg * B * d;
}

long long lru_blocks(int L, int B, int d) {
  return (long long)B * ((d + 63) / 64) * plan(L, B, d, true).nseg;  // one channel a lane
}

hipError_t lru_launch(const LruArgs& a, hipStream_t stream) {
  return dispatch(a, false, pairs_ok(a, [&](auto f) { f(a.x), f(a.r), f(a.i), f(a.h); }), stream);
}

hipError_t lru_grad_launch(const LruArgs& a, hipStream_t stream) {
  return dispatch(a, true, pairs_ok(a, [&](auto f) {
                    f(a.x), f(a.r), f(a.i), f(a.dh), f(a.dx), f(a.dr), f(a.di);
                  }), stream);
}

}  // namespace sru
