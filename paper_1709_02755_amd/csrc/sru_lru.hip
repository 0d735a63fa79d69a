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
// steps; both directions are one scan over such maps.  A wave holds kLruSteps
// steps of 64 lanes, VEC channels each, in registers, and a workgroup's waves,
// consecutive in time, a segment.  Their maps meet in LDS: each wave gets the state
// that enters its steps, runs them and writes.  A workgroup goes through the
// segments of its channels in turn and loads the next one while it finishes
// this one, so everything is read once.  Where that leaves most of the GPU idle
// (few channels, a long sequence), a sequence is cut into chunks of segments: one
// kernel folds all chunks but the last into their maps, and then each chunk's
// workgroup starts from the maps before it.  No workgroup waits for another one,
// and the results do not depend on when which one ran.
//
// What bounds it: memory, with the gates' arithmetic close behind (39 vector
// instructions an element forward, 5 of them exp, rcp or sqrt; the vector units are
// busy 46 % of the time forward, 50 % of the gradient's).  L 256, B 64, d 1024 in
// bf16, each call repeated by itself: 32 us for 134 MB (4.2 TB/s) and 61 us for 235
// MB (3.9), where a copy that moves as much makes 6.4; in a training step, forward
// and gradient in turn, the kernels take 36 and 52 + 5, the gradient's with part of
// its inputs still in the caches.  L 32768, B 1, d 1024: 110 us and 144 us (in turn 61
// + 63 and 35 + 111 + 5), for three quarters more to read forward and a third more
// in the gradient than in one pass; workgroups that handed on their state to the
// next one through memory read everything once, but took 114 and 171 us: a state
// needs 2 to 3 us from one workgroup to the next.
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
constexpr int kWaves = 8, kGradWaves = 4;          // of a workgroup
constexpr int kWideWaves = 16, kWideGradWaves = 8;  // of one with one channel a lane, unchunked
constexpr float kTiny = 1.17549435e-38f;
constexpr float kLog2e = 1.44269504088896341f;

__device__ __forceinline__ float exp2_hw(float x) { return __builtin_amdgcn_exp2f(x); }
// At least kTiny; a NaN stays one, which fmaxf would drop (v_maximum3_f32 here).
__device__ __forceinline__ float at_least_tiny(float x) {
  return __builtin_elementwise_maximum(x, kTiny);
}

struct Map {
  float A, B;
};
__device__ __forceinline__ float apply(Map m, float h) { return m.A == 0.f ? m.B : fmaf(m.A, h, m.B); }
// `late` after `early`.  (A NaN may leave A here, and where the steps' maps are
// made: a decay that is NaN has entered B as well.)
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

// A tensor's packed values at a wave's T steps from t0, zeros where there are none.
template <bool BF16, int VEC>
__device__ __forceinline__ void load_steps(const LruArgs& a, const Seq& s, const Lane& n, int t0,
                                           Pack<BF16, VEC> (&x)[T]) {
  const Ptr<BF16, VEC> p(s, n, t0);
#pragma unroll
  for (int u = 0; u < T; ++u) x[u] = Pack<BF16, VEC>{};
  if (!n.live) return;
  if (t0 + T <= a.L) {
#pragma unroll
    for (int u = 0; u < T; ++u) x[u] = p.load(u);
  } else {
#pragma unroll
    for (int u = 0; u < T; ++u)
      if (t0 + u < a.L) x[u] = p.load(u);
  }
}

// Lane u's marks of the wave's step u, as they are in memory.
struct Marks {
  unsigned pad, fresh;
};
template <bool FLAGS>
__device__ __forceinline__ Marks load_marks(const LruArgs& a, const Lane& n, int t0) {
  Marks m{0, 0};
  if constexpr (FLAGS) {
    const int u = threadIdx.x & 63;
    if (u < T && t0 + u < a.L) {
      const long long o = (long long)(t0 + u) * a.B + n.b;
      if (a.mask) m.pad = a.mask[o];
      if (a.reset) m.fresh = a.reset[o];
    }
  }
  return m;
}

// What a wave knows of its T steps: how many there are, and bit u of pad, fresh
// for step u.
struct Flags {
  int count;
  unsigned pad, fresh;
};
template <bool FLAGS>
__device__ __forceinline__ Flags flags_of(const LruArgs& a, int t0, const Marks& m) {
  Flags f{min(max(a.L - t0, 0), T), 0, 0};
  if constexpr (FLAGS) {
    f.pad = (unsigned)__ballot(m.pad != 0);
    f.fresh = (unsigned)__ballot(m.fresh != 0) & ~f.pad;
  }
  return f;
}

// Most waves of a call with marks have none of their own, or only padding: they
// take shorter ways (and the same values).
template <bool FLAGS>
__device__ __forceinline__ bool unmarked(const Flags& f) {
  return !FLAGS || (f.count == T && (f.pad | f.fresh) == 0);
}
template <bool FLAGS>
__device__ __forceinline__ bool all_padded(const Flags& f) {
  return FLAGS && f.pad == (1u << f.count) - 1;
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
  const float p = series(kept), e = at_least_tiny(exp2_hw(-kLog2e * kept));
  const bool small = kept < kSeriesEnd;
  const float w = small ? p : 1.f - e;
  return Decay{small ? 1.f - p : e, w * (2.f - w)};
}

// k = c softplus(lam) of a feature
__device__ __forceinline__ float decay_rate(const LruArgs& a, int j) {
  const float l = a.lam[j];
  return a.c * (fmaxf(l, 0.f) + log1pf(expf(-fabsf(l))));
}
// k of the lane's channels: the first wave works them out for all.  Returns
// whether all of the wave's series converge (s <= 1).
template <int VEC>
__device__ __forceinline__ bool decay_rates(const LruArgs& a, const Lane& n, float* lds,
                                            float (&k)[VEC]) {
  if (threadIdx.x < 64) {
#pragma unroll
    for (int v = 0; v < VEC; ++v)
      lds[v * 64 + threadIdx.x] = n.live ? decay_rate(a, n.j + v) : 0.f;
  }
  __syncthreads();
  bool beyond = false;
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    k[v] = lds[v * 64 + (threadIdx.x & 63)];
    beyond |= !(k[v] < kSeriesEnd);
  }
  return !__any(beyond);
}

// A segment is what a workgroup's waves hold at a time, a chunk the segments
// that one workgroup goes through, both counted in the order of the scan.
struct Cut {
  Map* maps;  // [chunks - 1, B * d]
  float* h0;  // [B * d], forward: what the chunks read as h0
  int nseg, each, chunks, groups;  // segments, those of a chunk, chunks, lane groups
};

// What the waves of a workgroup share: there are two sets of maps in turn, so
// that a segment takes one barrier.
template <int VEC, int W>
struct Shared {
  Map maps[2][W * VEC * 64];  // of the waves, in the order of the scan
  float rates[VEC * 64];
};

// Turns the state that enters the sequence into the one that enters the chunk, by
// the maps of the chunks before it: a wave joins a run of them, and all waves
// those joined.
template <int VEC, int W>
__device__ __forceinline__ void enter_chunk(const LruArgs& a, const Cut& c, const Lane& n,
                                            int chunk, Shared<VEC, W>& sh, float (&in)[VEC]) {
  if (chunk == 0) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int run = (chunk + W - 1) / W, last = min(chunk, (wave + 1) * run);
  const long long lanes = (long long)a.B * a.d;
  Map m[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) m[v] = Map{1.f, 0.f};
#pragma unroll 4
  for (int e = wave * run; e < last; ++e) {
#pragma unroll
    for (int v = 0; v < VEC; ++v)
      if (n.live) m[v] = join(c.maps[e * lanes + n.chan + v], m[v]);
  }
  if (wave * run < chunk) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) sh.maps[1][(wave * VEC + v) * 64 + lane] = m[v];
  }
  __syncthreads();
  for (int w = 0; w * run < chunk; ++w)
#pragma unroll
    for (int v = 0; v < VEC; ++v) in[v] = apply(sh.maps[1][(w * VEC + v) * 64 + lane], in[v]);
}

// The state that enters the wave's steps (`place` in the order of the scan) from
// the one that enters the segment, which becomes the next segment's.
template <int U, int VEC>
__device__ __forceinline__ void enter_wave(const Map* maps, int place, int waves,
                                           float (&seg_in)[VEC], float (&in)[VEC]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int v = 0; v < VEC; ++v) in[v] = seg_in[v];
#pragma unroll U
  for (int w = 0; w < waves; ++w)
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      if (w == place) in[v] = seg_in[v];
      seg_in[v] = apply(maps[(w * VEC + v) * 64 + lane], seg_in[v]);
    }
}

// A chunk's map, from those of the waves.
template <int VEC, int W>
__device__ __forceinline__ void chunk_map(const LruArgs& a, const Cut& c, const Lane& n, int chunk,
                                          int place, Shared<VEC, W>& sh, Map (&m)[VEC]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int v = 0; v < VEC; ++v) sh.maps[0][(place * VEC + v) * 64 + lane] = m[v];
  __syncthreads();
  if (place != 0 || !n.live) return;
#pragma unroll
  for (int w = 1; w < W; ++w)
#pragma unroll
    for (int v = 0; v < VEC; ++v) m[v] = join(sh.maps[0][(w * VEC + v) * 64 + lane], m[v]);
#pragma unroll
  for (int v = 0; v < VEC; ++v) c.maps[chunk * ((long long)a.B * a.d) + n.chan + v] = m[v];
}

// -------------------------------------------------------------------- forward
// A wave's steps as maps h -> A h + B (A of a document's first step is 0), and
// the map of them all.  FLAGS: some step may be missing, be padded or start a
// document.
template <bool FLAGS, bool SERIES, bool BF16, int VEC>
__device__ __forceinline__ void step_maps(const Pack<BF16, VEC> (&x)[T],
                                          const Pack<BF16, VEC> (&r)[T],
                                          const Pack<BF16, VEC> (&i)[T], const float (&k)[VEC],
                                          const Flags& f, float (&A)[T][VEC], float (&Bv)[T][VEC],
                                          Map (&all)[VEC]) {
#pragma unroll
  for (int v = 0; v < VEC; ++v) all[v] = Map{1.f, 0.f};
#pragma unroll
  for (int u = 0; u < T; ++u) {
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
template <bool FLAGS, bool BF16, int VEC>
__device__ __forceinline__ void run_steps(const LruArgs& a, const Lane& n, int t0, const Flags& f,
                                          const float (&A)[T][VEC], const float (&Bv)[T][VEC],
                                          float (&h)[VEC]) {
  const Ptr<BF16, VEC> out(a.h, n, t0);
  if (a.states) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) a.states[(long long)(t0 / T) * a.B * a.d + n.chan + v] = h[v];
  }
#pragma unroll
  for (int u = 0; u < T; ++u) {
    if (FLAGS && u >= f.count) continue;
    const bool pad = FLAGS && (f.pad >> u & 1), fresh = FLAGS && (f.fresh >> u & 1);
    float y[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      const float hn = fresh ? Bv[u][v] : fmaf(A[u][v], h[v], Bv[u][v]);
      h[v] = pad ? h[v] : hn;
      y[v] = pad ? 0.f : hn;
    }
    out.store(u, y);
  }
}

// A wave's way through its workgroup's segments: the loads of the next one are
// under way from when this one's values have been used.
template <bool FLAGS, bool SERIES, bool BF16, int VEC, int W>
__device__ __forceinline__ void lru_walk(const LruArgs& a, const Lane& n, int rank, int last,
                                         int wave, int waves, const float (&k)[VEC],
                                         float (&seg_in)[VEC], Pack<BF16, VEC> (&x)[T],
                                         Pack<BF16, VEC> (&r)[T],
                                         Pack<BF16, VEC> (&i)[T], Marks marks,
                                         Shared<VEC, W>& sh) {
  int set = 0;
#pragma unroll 1
  for (; rank < last; ++rank, set ^= 1) {
    const int t0 = (rank * waves + wave) * T;
    const Flags f = flags_of<FLAGS>(a, t0, marks);
    float A[T][VEC], Bv[T][VEC], h[VEC];
    Map m[VEC];
    if (unmarked<FLAGS>(f)) {
      step_maps<false, SERIES, BF16, VEC>(x, r, i, k, f, A, Bv, m);
    } else if (all_padded<FLAGS>(f)) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) m[v] = Map{1.f, 0.f};
    } else {
      step_maps<FLAGS, SERIES, BF16, VEC>(x, r, i, k, f, A, Bv, m);
    }
#pragma unroll
    for (int v = 0; v < VEC; ++v) sh.maps[set][(wave * VEC + v) * 64 + (threadIdx.x & 63)] = m[v];
    if (rank + 1 < last) {
      const int t1 = t0 + waves * T;
      load_steps<BF16, VEC>(a, a.r, n, t1, r);
      load_steps<BF16, VEC>(a, a.i, n, t1, i);
      load_steps<BF16, VEC>(a, a.x, n, t1, x);
      marks = load_marks<FLAGS>(a, n, t1);
    }
    __syncthreads();
    enter_wave<4>(sh.maps[set], wave, waves, seg_in, h);
    if (n.live && f.count) {
      if (unmarked<FLAGS>(f))
        run_steps<false, BF16, VEC>(a, n, t0, f, A, Bv, h);
      else
        run_steps<FLAGS, BF16, VEC>(a, n, t0, f, A, Bv, h);
      if (a.h_last && t0 + T >= a.L) {
#pragma unroll
        for (int v = 0; v < VEC; ++v) a.h_last[n.chan + v] = h[v];
      }
    }
  }
}

// FLAGS: there is padding or a new document somewhere, or a wave's last steps
// are missing.  All waves of a workgroup have the same channels, so all take
// the same body.
template <bool BF16, int VEC, bool FLAGS, int W>
__global__ __launch_bounds__(64 * W, 4) void lru_kernel(LruArgs a, Cut c) {
  __shared__ Shared<VEC, W> sh;
  const int group = blockIdx.x % (unsigned)c.groups, chunk = blockIdx.x / (unsigned)c.groups;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const Lane n = lane_of<VEC>(a, group);
  const int rank = chunk * c.each, last = min(rank + c.each, c.nseg);
  const int t0 = (rank * waves + wave) * T;
  Pack<BF16, VEC> x[T], r[T], i[T];
  load_steps<BF16, VEC>(a, a.r, n, t0, r);
  load_steps<BF16, VEC>(a, a.i, n, t0, i);
  load_steps<BF16, VEC>(a, a.x, n, t0, x);
  const Marks marks = load_marks<FLAGS>(a, n, t0);
  float k[VEC], in[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) in[v] = a.h0 && n.live ? a.h0[n.chan + v] : 0.f;
  enter_chunk(a, c, n, chunk, sh, in);
  if (decay_rates<VEC>(a, n, sh.rates, k))
    lru_walk<FLAGS, true, BF16, VEC, W>(a, n, rank, last, wave, waves, k, in, x, r, i, marks, sh);
  else
    lru_walk<FLAGS, false, BF16, VEC, W>(a, n, rank, last, wave, waves, k, in, x, r, i, marks, sh);
}

// The maps of all chunks but the last: a wave has its steps in a row.
template <bool FLAGS, bool SERIES, bool BF16, int VEC>
__device__ __forceinline__ void run_map(const LruArgs& a, const Lane& n, int t0, int count,
                                        const float (&k)[VEC], Map (&m)[VEC]) {
#pragma unroll
  for (int v = 0; v < VEC; ++v) m[v] = Map{1.f, 0.f};
#pragma unroll 1
  for (int q = 0; q < count; ++q, t0 += T) {
    Pack<BF16, VEC> x[T], r[T], i[T];
    load_steps<BF16, VEC>(a, a.r, n, t0, r);
    load_steps<BF16, VEC>(a, a.i, n, t0, i);
    load_steps<BF16, VEC>(a, a.x, n, t0, x);
    const Flags f = flags_of<FLAGS>(a, t0, load_marks<FLAGS>(a, n, t0));
    if (all_padded<FLAGS>(f)) continue;
    float A[T][VEC], Bv[T][VEC];
    Map one[VEC];
    if (unmarked<FLAGS>(f))
      step_maps<false, SERIES, BF16, VEC>(x, r, i, k, f, A, Bv, one);
    else
      step_maps<FLAGS, SERIES, BF16, VEC>(x, r, i, k, f, A, Bv, one);
#pragma unroll
    for (int v = 0; v < VEC; ++v) m[v] = join(one[v], m[v]);
  }
}
template <bool BF16, int VEC, bool FLAGS, int W>
__global__ __launch_bounds__(64 * W, 5) void lru_maps_kernel(LruArgs a, Cut c) {
  __shared__ Shared<VEC, W> sh;
  const int group = blockIdx.x % (unsigned)c.groups, chunk = blockIdx.x / (unsigned)c.groups;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Lane n = lane_of<VEC>(a, group);
  const int t0 = (chunk * W + wave) * c.each * T;
  // h_last may be h0's own memory, and the last chunk writes it while others may
  // not have started: they read a copy, made before any of them runs
  if (a.h0 && chunk == 0 && wave == 0 && n.live) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) c.h0[n.chan + v] = a.h0[n.chan + v];
  }
  float k[VEC];
  Map m[VEC];
  if (decay_rates<VEC>(a, n, sh.rates, k))
    run_map<FLAGS, true, BF16, VEC>(a, n, t0, c.each, k, m);
  else
    run_map<FLAGS, false, BF16, VEC>(a, n, t0, c.each, k, m);
  chunk_map(a, c, n, chunk, wave, sh, m);
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
      const float q = at_least_tiny(dc.q);
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

template <bool FLAGS, bool SERIES, bool BF16, int VEC, int W>
__device__ __forceinline__ void grad_walk(const LruArgs& a, const Lane& n, int nseg, int rank,
                                          int last, int wave, int waves, const float (&k)[VEC],
                                          float (&seg_in)[VEC], float (&h)[VEC],
                                          Pack<BF16, VEC> (&x)[T], Pack<BF16, VEC> (&r)[T],
                                          Pack<BF16, VEC> (&i)[T], Pack<BF16, VEC> (&dh)[T],
                                          Marks marks, Shared<VEC, W>& sh, float (&acc)[VEC]) {
  const int place = waves - 1 - wave, lane = threadIdx.x & 63;
#pragma unroll
  for (int v = 0; v < VEC; ++v) acc[v] = 0.f;
  int set = 0;
#pragma unroll 1
  for (; rank < last; ++rank, set ^= 1) {
    const int t0 = ((nseg - 1 - rank) * waves + wave) * T;
    const Flags f = flags_of<FLAGS>(a, t0, marks);
    GradSteps<VEC> st;
    Map m[VEC];
    if (all_padded<true>(f)) {  // or without a step
#pragma unroll
      for (int v = 0; v < VEC; ++v) m[v] = Map{1.f, 0.f};
    } else if (unmarked<FLAGS>(f)) {
      grad_maps<false, SERIES, BF16, VEC>(x, r, i, dh, k, f, h, st, m);
    } else {
      grad_maps<FLAGS, SERIES, BF16, VEC>(x, r, i, dh, k, f, h, st, m);
    }
#pragma unroll
    for (int v = 0; v < VEC; ++v) sh.maps[set][(place * VEC + v) * 64 + lane] = m[v];
    Pack<BF16, VEC> now[T];
#pragma unroll
    for (int u = 0; u < T; ++u) now[u] = dh[u];
    if (rank + 1 < last) {
      const int t1 = t0 - waves * T;
      load_steps<BF16, VEC>(a, a.r, n, t1, r);
      load_steps<BF16, VEC>(a, a.dh, n, t1, dh);
      load_steps<BF16, VEC>(a, a.i, n, t1, i);
      load_steps<BF16, VEC>(a, a.x, n, t1, x);
      marks = load_marks<FLAGS>(a, n, t1);
#pragma unroll
      for (int v = 0; v < VEC; ++v)
        h[v] = n.live ? a.states[(long long)(t1 / T) * a.B * a.d + n.chan + v] : 0.f;
    }
    __syncthreads();
    float carry[VEC];
    enter_wave<1>(sh.maps[set], place, waves, seg_in, carry);
    if (n.live && f.count) {
      if (unmarked<FLAGS>(f))
        grad_steps<false, BF16, VEC>(a, n, t0, now, st, f, carry, acc);
      else
        grad_steps<FLAGS, BF16, VEC>(a, n, t0, now, st, f, carry, acc);
      if (a.dh0 && t0 == 0) {
#pragma unroll
        for (int v = 0; v < VEC; ++v) a.dh0[n.chan + v] = carry[v];
      }
    }
  }
}

// The scan runs from the last step to the first: rank 0 is the last segment,
// and a workgroup's last wave comes first.  sums: [chunks, B, d] of -sum dla s.
template <bool BF16, int VEC, bool FLAGS, int W>
__global__ __launch_bounds__(64 * W, VEC == 1 ? 3 : 2) void lru_grad_kernel(LruArgs a, Cut c, float* sums) {
  __shared__ Shared<VEC, W> sh;
  const int group = blockIdx.x % (unsigned)c.groups, chunk = blockIdx.x / (unsigned)c.groups;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const Lane n = lane_of<VEC>(a, group);
  const int rank = chunk * c.each, last = min(rank + c.each, c.nseg);
  const int t0 = ((c.nseg - 1 - rank) * waves + wave) * T;
  Pack<BF16, VEC> x[T], r[T], i[T], dh[T];
  load_steps<BF16, VEC>(a, a.r, n, t0, r);
  load_steps<BF16, VEC>(a, a.dh, n, t0, dh);
  load_steps<BF16, VEC>(a, a.i, n, t0, i);
  load_steps<BF16, VEC>(a, a.x, n, t0, x);
  const Marks marks = load_marks<FLAGS>(a, n, t0);
  float k[VEC], in[VEC], h[VEC], acc[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    in[v] = a.dh_last && n.live ? a.dh_last[n.chan + v] : 0.f;
    h[v] = n.live && t0 < a.L ? a.states[(long long)(t0 / T) * a.B * a.d + n.chan + v] : 0.f;
  }
  enter_chunk(a, c, n, chunk, sh, in);
  if (decay_rates<VEC>(a, n, sh.rates, k))
    grad_walk<FLAGS, true, BF16, VEC, W>(a, n, c.nseg, rank, last, wave, waves, k, in, h, x, r, i,
                                         dh, marks, sh, acc);
  else
    grad_walk<FLAGS, false, BF16, VEC, W>(a, n, c.nseg, rank, last, wave, waves, k, in, h, x, r, i,
                                          dh, marks, sh, acc);

  // the waves' sums in a fixed order
  float* red = reinterpret_cast<float*>(sh.maps);
  const int lane = threadIdx.x & 63;
  __syncthreads();
#pragma unroll
  for (int v = 0; v < VEC; ++v) red[(wave * VEC + v) * 64 + lane] = acc[v];
  __syncthreads();
  if (wave == 0 && n.live) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      float t = acc[v];
      for (int q = 1; q < waves; ++q) t += red[(q * VEC + v) * 64 + lane];
      sums[chunk * ((long long)a.B * a.d) + n.chan + v] = t;
    }
  }
}

// The map of grad_maps alone.
template <bool FLAGS, bool SERIES, bool BF16, int VEC>
__device__ __forceinline__ void grad_map(const Pack<BF16, VEC> (&r)[T],
                                         const Pack<BF16, VEC> (&dh)[T], const float (&k)[VEC],
                                         const Flags& f, Map (&all)[VEC]) {
#pragma unroll
  for (int v = 0; v < VEC; ++v) all[v] = Map{1.f, 0.f};
#pragma unroll
  for (int u = 0; u < T; ++u) {
    const bool pad = FLAGS && ((f.pad >> u & 1) || u >= f.count);
    const bool cut = FLAGS && (f.fresh & (2u << u) - 1) != 0;
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      const Decay dc = decay_of<SERIES>(decay_kept<SERIES>(k[v], sigmoid_fast(r[u].get(v))));
      const float A = all[v].A * dc.a;
      const float B = fmaf(A, dh[u].get(v), all[v].B);
      all[v].A = pad ? all[v].A : A;
      all[v].B = pad || cut ? all[v].B : B;
    }
  }
  const bool anew = FLAGS && f.fresh != 0;
#pragma unroll
  for (int v = 0; v < VEC; ++v) all[v].A = anew ? 0.f : fmaxf(all[v].A, kTiny);
}

// The maps of the carried gradient of all chunks but the last in the order of the
// scan, by r and dh alone.
template <bool FLAGS, bool SERIES, bool BF16, int VEC>
__device__ __forceinline__ void grad_run_map(const LruArgs& a, const Lane& n, int t0, int count,
                                             const float (&k)[VEC], Map (&m)[VEC]) {
#pragma unroll
  for (int v = 0; v < VEC; ++v) m[v] = Map{1.f, 0.f};
  t0 += (count - 1) * T;
#pragma unroll 1
  for (int q = 0; q < count; ++q, t0 -= T) {
    Pack<BF16, VEC> r[T], dh[T];
    load_steps<BF16, VEC>(a, a.r, n, t0, r);
    load_steps<BF16, VEC>(a, a.dh, n, t0, dh);
    const Flags f = flags_of<FLAGS>(a, t0, load_marks<FLAGS>(a, n, t0));
    if (all_padded<true>(f)) continue;  // or without a step
    Map one[VEC];
    if (unmarked<FLAGS>(f))
      grad_map<false, SERIES, BF16, VEC>(r, dh, k, f, one);
    else
      grad_map<FLAGS, SERIES, BF16, VEC>(r, dh, k, f, one);
#pragma unroll
    for (int v = 0; v < VEC; ++v) m[v] = join(one[v], m[v]);
  }
}
template <bool BF16, int VEC, bool FLAGS, int W>
__global__ __launch_bounds__(64 * W, 5) void lru_grad_maps_kernel(LruArgs a, Cut c) {
  __shared__ Shared<VEC, W> sh;
  const int group = blockIdx.x % (unsigned)c.groups, chunk = blockIdx.x / (unsigned)c.groups;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Lane n = lane_of<VEC>(a, group);
  // the chunk's first segment in time
  const int first = c.nseg - (chunk + 1) * c.each;
  const int t0 = (first * W + wave * c.each) * T;
  float k[VEC];
  Map m[VEC];
  if (decay_rates<VEC>(a, n, sh.rates, k))
    grad_run_map<FLAGS, true, BF16, VEC>(a, n, t0, c.each, k, m);
  else
    grad_run_map<FLAGS, false, BF16, VEC>(a, n, t0, c.each, k, m);
  chunk_map(a, c, n, chunk, W - 1 - wave, sh, m);
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

// How a call is cut, by its groups of 64 channels of a sequence (us, bf16, forward
// and gradient, each call repeated by itself on one box):
// - many: two channels a lane, small workgroups, which overlap each other's loads
//   and arithmetic.  L 256, B 64, d 1024 (1,024 groups): 32 / 61; workgroups of 16
//   and 8 waves of one channel a lane 44 / 70.
// - fewer, or few steps: one channel a lane, so twice the workgroups, and large
//   ones.  L 1024, B 16, d 1024 (256 groups): 38 / 65, as chunks 56 / 74; L 200,
//   B 16, d 256: 11.7 / 19.2, as chunks 15.5 / 22.  L 256, B 32, d 1024 (512
//   groups): the forward, whose small workgroups have eight waves, takes 19 with
//   two channels a lane and 22 so; L 512, B 48, d 1024 the gradient 101 and 94.
// - few groups, many steps: chunks, so many that there are about 512 workgroups of
//   two channels a lane.  L 32768, B 1, d 1024 (16 groups): 110 / 143; as many
//   chunks of one channel a lane 127 / 149; L 8192, B 8, d 1024 (128 groups): 206 /
//   260, without chunks 236 / 359.
constexpr long long kMany = 512, kGradMany = 1024, kFew = 256, kChunked = 1024, kMostChunks = 256;
constexpr int kWideRounds = 4;
struct Plan {
  bool wide;                      // large workgroups of one channel a lane
  int waves, nseg, each, chunks;  // of a workgroup, segments, those of a chunk, chunks
};
// Groups of one channel a lane; d may be any int, for the check of the sizes.
long long lane_groups(int B, int d) { return B * ((d + 63LL) / 64); }
Plan plan(int L, int B, int d, bool grad) {
  const int n = (L + T - 1) / T;
  const long long groups = lane_groups(B, d);
  const int wide = grad ? kWideGradWaves : kWideWaves;
  Plan p;
  p.wide = groups < (grad ? kGradMany : kMany) && (groups >= kFew || n <= kWideRounds * wide);
  const int most = p.wide ? wide : grad ? kGradWaves : kWaves;
  p.nseg = (n + most - 1) / most;
  p.waves = (n + p.nseg - 1) / p.nseg;
  p.each = p.nseg, p.chunks = 1;
  if (!p.wide && groups < kFew) {
    const long long want = std::min({(kChunked + groups - 1) / groups, (long long)p.nseg, kMostChunks});
    p.waves = most;
    p.each = (int)((p.nseg + want - 1) / want);
    p.chunks = (p.nseg + p.each - 1) / p.each;
  }
  return p;
}

// Two channels of 16 bits a lane, where every pair of features lies on its size.
template <typename F>
bool pairs_ok(const LruArgs& a, F each) {
  if (a.d & 1) return false;
  bool ok = true;
  each([&](const Seq& s) {
    ok = ok && ((reinterpret_cast<uintptr_t>(s.p) & 3) == 0) && !(s.st & 1) && !(s.sb & 1);
  });
  return ok;
}

size_t align_up(size_t x) { return (x + 255) / 256 * 256; }
template <bool BF16, int VEC, bool FLAGS, bool WIDE>
hipError_t launch(LruArgs a, const Cut& c, const Plan& p, hipStream_t st) {
  constexpr int W = WIDE ? kWideWaves : kWaves;
  if constexpr (!WIDE) {
    if (c.chunks > 1) {
      timing_before("lru_maps", st);
      hipLaunchKernelGGL((lru_maps_kernel<BF16, VEC, FLAGS, W>),
                         dim3((unsigned)c.groups * (c.chunks - 1)), dim3(64 * W), 0, st, a, c);
      timing_after(st);
      if (hipError_t e = hipGetLastError()) return e;
      if (a.h0) a.h0 = c.h0;
    }
  }
  timing_before("lru", st);
  hipLaunchKernelGGL((lru_kernel<BF16, VEC, FLAGS, W>), dim3((unsigned)c.groups * c.chunks),
                     dim3(64 * p.waves), 0, st, a, c);
  timing_after(st);
  return hipGetLastError();
}
template <bool BF16, int VEC, bool FLAGS, bool WIDE>
hipError_t launch_grad(const LruArgs& a, const Cut& c, const Plan& p, float* sums, hipStream_t st) {
  constexpr int W = WIDE ? kWideGradWaves : kGradWaves;
  if constexpr (!WIDE) {
    if (c.chunks > 1) {
      timing_before("lru_grad_maps", st);
      hipLaunchKernelGGL((lru_grad_maps_kernel<BF16, VEC, FLAGS, W>),
                         dim3((unsigned)c.groups * (c.chunks - 1)), dim3(64 * W), 0, st, a, c);
      timing_after(st);
      if (hipError_t e = hipGetLastError()) return e;
    }
  }
  timing_before("lru_grad", st);
  hipLaunchKernelGGL((lru_grad_kernel<BF16, VEC, FLAGS, W>), dim3((unsigned)c.groups * c.chunks),
                     dim3(64 * p.waves), 0, st, a, c, sums);
  timing_after(st);
  if (hipError_t e = hipGetLastError()) return e;
  timing_before("lru_sums", st);
  hipLaunchKernelGGL(lru_sums_kernel, dim3((a.d + 63) / 64), dim3(1024), 0, st, a, sums,
                     (long long)c.chunks * a.B);
  timing_after(st);
  return hipGetLastError();
}

// Workspace: the chunks' maps, then the state that enters (forward, where there
// are chunks) or the sums (gradient).
size_t maps_bytes(const Plan& p, int B, int d) {
  return align_up(sizeof(Map) * (size_t)(p.chunks - 1) * B * d);
}

template <bool BF16, int VEC, bool WIDE>
hipError_t run(const LruArgs& a, const Plan& p, bool grad, hipStream_t st) {
  float* rest = reinterpret_cast<float*>(static_cast<char*>(a.workspace) + maps_bytes(p, a.B, a.d));
  const Cut c{static_cast<Map*>(a.workspace), rest, p.nseg, p.each, p.chunks,
              a.B * ((a.d + 64 * VEC - 1) / (64 * VEC))};
  const bool flags = a.mask || a.reset || a.L % T;
  if (grad)
    return flags ? launch_grad<BF16, VEC, true, WIDE>(a, c, p, rest, st)
                 : launch_grad<BF16, VEC, false, WIDE>(a, c, p, rest, st);
  return flags ? launch<BF16, VEC, true, WIDE>(a, c, p, st)
               : launch<BF16, VEC, false, WIDE>(a, c, p, st);
}

hipError_t dispatch(const LruArgs& a, bool grad, bool pairs, hipStream_t st) {
  const Plan p = plan(a.L, a.B, a.d, grad);
  if (!a.bf16)
    return p.wide ? run<false, 1, true>(a, p, grad, st) : run<false, 1, false>(a, p, grad, st);
  if (p.wide) return run<true, 1, true>(a, p, grad, st);
  return pairs ? run<true, 2, false>(a, p, grad, st) : run<true, 1, false>(a, p, grad, st);
}

}  // namespace

size_t lru_workspace_bytes(int L, int B, int d) {
  const Plan p = plan(L, B, d, false);
  return p.chunks == 1 ? 0 : maps_bytes(p, B, d) + sizeof(float) * (size_t)B * d;
}

size_t lru_grad_workspace_bytes(int L, int B, int d) {
  const Plan p = plan(L, B, d, true);
  return maps_bytes(p, B, d) + sizeof(float) * (size_t)p.chunks * B * d;
}

long long lru_blocks(int L, int B, int d) {
  return lane_groups(B, d) * std::max(plan(L, B, d, false).chunks, plan(L, B, d, true).chunks);
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
