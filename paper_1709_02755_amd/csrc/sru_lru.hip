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
// steps of 64 lanes (VEC channels each) in registers, a workgroup up to 16
// waves, consecutive in time: a segment.  Maps are joined in the workgroup
// through LDS and, where a sequence has several segments, across workgroups
// through one 64-bit word per channel and segment: everything is read once.
//
// A map with A = 0 forgets what came before: that is how a new document's
// start, and a state that is known, are written (a state of NaN before a new
// document must not reach it through 0 * NaN).  Products of decays that are
// merely small stay above 0.
#include "sru_device.h"
#include "sru_lm.h"

namespace sru {
namespace {

constexpr int T = kLruSteps;
constexpr int kWaves = 16;             // waves of a full workgroup
constexpr int kSegment = kWaves * T;   // its steps
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

// Where a lane's channels lie.
struct Lane {
  bool live;
  int b, j;         // sequence, first feature
  long long chan;   // b * d + j
};
template <int VEC>
__device__ __forceinline__ Lane lane_of(const LruArgs& a, int group) {
  const int per = a.d / VEC;
  const long long l = (long long)group * 64 + (threadIdx.x & 63);
  Lane n;
  n.live = l < (long long)a.B * per;
  const long long ll = n.live ? l : 0;
  n.b = (int)(ll / per);
  n.j = (int)(ll - (long long)n.b * per) * VEC;
  n.chan = (long long)n.b * a.d + n.j;
  return n;
}

template <bool BF16, int VEC>
__device__ __forceinline__ const Pack<BF16, VEC>* at(const Seq& s, const Lane& n, int t) {
  constexpr int ES = BF16 ? 2 : 4;
  return reinterpret_cast<const Pack<BF16, VEC>*>(static_cast<const char*>(s.p) +
                                                  ES * (t * s.st + n.b * s.sb + n.j));
}
template <bool BF16, int VEC>
__device__ __forceinline__ Pack<BF16, VEC>* out_at(const Seq& s, const Lane& n, int t) {
  return const_cast<Pack<BF16, VEC>*>(at<BF16, VEC>(s, n, t));
}

// What a wave knows of its steps: bit u of pad, fresh for step u.  Steps past
// the sequence's end are padded and out of range.
struct Flags {
  unsigned pad = 0, fresh = 0;
};
template <bool FLAGS>
__device__ __forceinline__ Flags flags_of(const LruArgs& a, const Lane& n, int t0) {
  Flags f;
  if constexpr (FLAGS) {
#pragma unroll
    for (int u = 0; u < T; ++u) {
      const int t = t0 + u;
      if (t >= a.L) break;
      const long long o = (long long)t * a.B + n.b;
      if (a.mask && a.mask[o]) f.pad |= 1u << u;
      if (a.reset && a.reset[o]) f.fresh |= 1u << u;
    }
    f.fresh &= ~f.pad;
  }
  const int left = a.L - t0;
  if (left < T) f.pad |= left <= 0 ? ~0u : ~0u << left;
  return f;
}

// A step's decay a = e^-y and q = 1 - a^2 from y = k s.  Both come from w = 1 -
// a, by the series of 1 - e^-y where that would cancel (its next term is y^7 /
// 5040, below 2^-24 of w here): q = w (2 - w), and a = 1 - w is rounded once, to
// nearest.  A state carried on over a thousand steps multiplies as many decays
// near 1: the error of the hardware's 2^x there, which leans to one side, would
// add up.
struct Decay {
  float a, q;
};
__device__ __forceinline__ Decay decay(float k, float s) {
  const float y = k * s;
  float p = fmaf(y, 1.f / 720.f, -1.f / 120.f);
  p = fmaf(y, p, 1.f / 24.f);
  p = fmaf(y, p, -1.f / 6.f);
  p = fmaf(y, p, 0.5f);
  p = fmaf(y, -p, 1.f) * y;
  const bool small = y < 0.25f;
  const float e = fmaxf(exp2_hw(-kLog2e * y), kTiny);
  const float w = small ? p : 1.f - e;
  // q at least the smallest number: its root's reciprocal is finite
  return Decay{small ? 1.f - p : e, fmaxf(w * (2.f - w), kTiny)};
}

// k of the lane's channels, worked out by the first wave
template <int VEC>
__device__ __forceinline__ void decay_rates(const LruArgs& a, const Lane& n, float* lds,
                                            float (&k)[VEC]) {
  if (threadIdx.x < 64) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      const float l = a.lam[n.j + v];
      const float sp = fmaxf(l, 0.f) + log1pf(expf(-fabsf(l)));
      lds[v * 64 + threadIdx.x] = a.c * sp;
    }
  }
  __syncthreads();
#pragma unroll
  for (int v = 0; v < VEC; ++v) k[v] = lds[v * 64 + (threadIdx.x & 63)];
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
  unsigned* ticket;
  unsigned long long* words;  // [nseg, B * d]
  int nseg, groups;
};

// A workgroup's place: tickets are handed out in the order in which workgroups
// start, and a segment only waits for those with lower tickets.  These have
// started, so they get on whatever else waits: every wait ends.
__device__ __forceinline__ unsigned take_ticket(const Chain& c, unsigned* lds) {
  if (c.nseg == 1) return blockIdx.x;
  if (threadIdx.x == 0)
    *lds = __hip_atomic_fetch_add(c.ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  __syncthreads();
  return *lds;
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

// The state that enters segment `rank` (> 0): each wave takes the map of one
// of the segments before it, the nearest first, and all join them, until none
// depends on what is still further back.  The segment of rank 0 leaves its
// state, so that is the last at the latest.  win: kWaves * 64 * VEC maps.
template <int VEC>
__device__ __forceinline__ void look_back(const Chain& c, const LruArgs& a, const Lane& n,
                                          int rank, Map* win, float (&in)[VEC]) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  Map m[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) m[v] = Map{1.f, 0.f};
  for (int last = rank - 1; last >= 0; last -= kWaves) {
    const int p = last - wave;
    Map got[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) got[v] = Map{1.f, 0.f};
    if (p >= 0 && n.live) {
      const unsigned long long* w = c.words + (long long)p * a.B * a.d + n.chan;
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        unsigned long long x = kEmpty;
        // the wait ends by the order of the tickets; the bound (seconds)
        // keeps a mistake there from hanging the GPU: the result is NaN then
        for (int spin = 0; spin < (1 << 22); ++spin) {
          x = __hip_atomic_load(w + v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
          if (x != kEmpty) break;
          __builtin_amdgcn_s_sleep(1);
        }
        got[v] = map_of(x);
      }
    }
    __syncthreads();  // win's earlier use is over
#pragma unroll
    for (int v = 0; v < VEC; ++v) win[(wave * VEC + v) * 64 + lane] = got[v];
    __syncthreads();
    bool open = false;
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      for (int w = 0; w < kWaves && w <= last; ++w) m[v] = join(m[v], win[(w * VEC + v) * 64 + lane]);
      open |= m[v].A != 0.f;
    }
    // every wave has the same maps, so all leave together
    if (!__any(open && n.live)) break;
  }
#pragma unroll
  for (int v = 0; v < VEC; ++v) in[v] = m[v].B;
}

// The maps of a workgroup's waves, in LDS in the order of the scan (`place` of
// a wave's steps in it), joined: the state that enters the wave's steps, and
// the segment's map where the state entering that is not known yet.
template <int VEC>
__device__ __forceinline__ void enter_wave(const Map* maps, int place, const float (&seg_in)[VEC],
                                           float (&in)[VEC]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    float h = seg_in[v];
    for (int w = 0; w < place; ++w) h = apply(maps[(w * VEC + v) * 64 + lane], h);
    in[v] = h;
  }
}

// Joins the waves' maps, publishes the segment's, waits for the state entering
// it and publishes the one that leaves.  first: what enters rank 0.
template <int VEC>
__device__ __forceinline__ void join_segments(const Chain& c, const LruArgs& a, const Lane& n,
                                              int rank, int waves, const Map* maps, Map* win,
                                              const float (&first)[VEC], float (&seg_in)[VEC]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int v = 0; v < VEC; ++v) seg_in[v] = first[v];
  if (c.nseg == 1) return;
  Map seg[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    seg[v] = maps[v * 64 + lane];
    for (int w = 1; w < waves; ++w) seg[v] = join(maps[(w * VEC + v) * 64 + lane], seg[v]);
  }
  const bool first_wave = threadIdx.x < 64, not_last = rank + 1 < c.nseg;
  if (rank > 0) {
    if (first_wave && not_last) publish<VEC>(c, a, n, rank, seg);
    look_back<VEC>(c, a, n, rank, win, seg_in);
  }
  if (first_wave && not_last) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) seg[v] = Map{0.f, apply(seg[v], seg_in[v])};
    publish<VEC>(c, a, n, rank, seg);
  }
}

__global__ __launch_bounds__(256) void lru_clear_kernel(unsigned* ticket,
                                                        unsigned long long* words, long long n) {
  const long long step = (long long)gridDim.x * 256;
  const long long first = (long long)blockIdx.x * 256 + threadIdx.x;
  if (first == 0) *ticket = 0;
  for (long long i = first; i < n; i += step) words[i] = kEmpty;
}

// -------------------------------------------------------------------- forward
template <bool BF16, int VEC, bool FLAGS>
__global__ __launch_bounds__(64 * kWaves) void lru_kernel(LruArgs a, Chain c) {
  __shared__ Map maps[kWaves * VEC * 64], win[kWaves * VEC * 64];
  __shared__ float rates[VEC * 64];
  __shared__ unsigned ticket;
  const unsigned id = take_ticket(c, &ticket);
  const int rank = id / c.groups, group = id - rank * c.groups;
  const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const Lane n = lane_of<VEC>(a, group);
  const int t0 = (rank * waves + wave) * T;

  Pack<BF16, VEC> x[T], r[T], i[T];
#pragma unroll
  for (int u = 0; u < T; ++u) {
    const int t = t0 + u;
    x[u] = r[u] = i[u] = Pack<BF16, VEC>{};
    if (t < a.L && n.live) {
      x[u] = *at<BF16, VEC>(a.x, n, t);
      r[u] = *at<BF16, VEC>(a.r, n, t);
      i[u] = *at<BF16, VEC>(a.i, n, t);
    }
  }
  const Flags f = flags_of<FLAGS>(a, n, t0);
  float k[VEC], first[VEC];
  decay_rates<VEC>(a, n, rates, k);
#pragma unroll
  for (int v = 0; v < VEC; ++v) first[v] = a.h0 && n.live ? a.h0[n.chan + v] : 0.f;

  float A[T][VEC], Bv[T][VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    Map m{1.f, 0.f};
    bool fresh = false;
#pragma unroll
    for (int u = 0; u < T; ++u) {
      const float s = sigmoid_fast(r[u].get(v)), g = sigmoid_fast(i[u].get(v));
      const Decay dc = decay(k[v], s);
      const float gx = g * x[u].get(v);
      float at = dc.a, bt = __builtin_amdgcn_sqrtf(dc.q) * gx;
      if (f.pad >> u & 1) at = 1.f, bt = 0.f;
      if (FLAGS && (f.fresh >> u & 1)) at = 0.f, bt = gx, fresh = true;
      A[u][v] = at;
      Bv[u][v] = bt;
      m.A *= at;
      m.B = at == 0.f ? bt : fmaf(at, m.B, bt);
    }
    m.A = fresh ? 0.f : fmaxf(m.A, kTiny);
    maps[(wave * VEC + v) * 64 + lane] = m;
  }
  __syncthreads();
  float seg_in[VEC], h[VEC];
  join_segments<VEC>(c, a, n, rank, waves, maps, win, first, seg_in);
  enter_wave<VEC>(maps, wave, seg_in, h);
  if (!n.live || t0 >= a.L) return;

  if (a.states) {
    float* p = a.states + (long long)(t0 / T) * a.B * a.d + n.chan;
#pragma unroll
    for (int v = 0; v < VEC; ++v) p[v] = h[v];
  }
#pragma unroll
  for (int u = 0; u < T; ++u) {
    const int t = t0 + u;
    float y[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      h[v] = apply(Map{A[u][v], Bv[u][v]}, h[v]);
      y[v] = (f.pad >> u & 1) ? 0.f : h[v];
    }
    if (t < a.L) {
      Pack<BF16, VEC> o;
      o.put(y);
      *out_at<BF16, VEC>(a.h, n, t) = o;
    }
  }
  if (a.h_last && t0 + T >= a.L) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) a.h_last[n.chan + v] = h[v];
  }
}

// ------------------------------------------------------------------- gradient
// The scan runs from the last step to the first: rank 0 is the last segment,
// and a workgroup's last wave comes first.  sums: [nseg, B, d] of -sum dla s.
template <bool BF16, int VEC, bool FLAGS>
__global__ __launch_bounds__(64 * kWaves) void lru_grad_kernel(LruArgs a, Chain c, float* sums) {
  __shared__ Map maps[kWaves * VEC * 64], win[kWaves * VEC * 64];
  __shared__ float rates[VEC * 64];
  __shared__ unsigned ticket;
  const unsigned id = take_ticket(c, &ticket);
  const int rank = id / c.groups, group = id - rank * c.groups;
  const int waves = blockDim.x >> 6, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int seg = c.nseg - 1 - rank;
  const Lane n = lane_of<VEC>(a, group);
  const int t0 = (seg * waves + wave) * T;

  Pack<BF16, VEC> x[T], r[T], i[T], dh[T];
#pragma unroll
  for (int u = 0; u < T; ++u) {
    const int t = t0 + u;
    x[u] = r[u] = i[u] = dh[u] = Pack<BF16, VEC>{};
    if (t < a.L && n.live) {
      r[u] = *at<BF16, VEC>(a.r, n, t);
      dh[u] = *at<BF16, VEC>(a.dh, n, t);
      x[u] = *at<BF16, VEC>(a.x, n, t);
      i[u] = *at<BF16, VEC>(a.i, n, t);
    }
  }
  const Flags f = flags_of<FLAGS>(a, n, t0);
  float k[VEC], first[VEC], h[VEC];
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    first[v] = a.dh_last && n.live ? a.dh_last[n.chan + v] : 0.f;
    h[v] = n.live && t0 < a.L ? a.states[(long long)(t0 / T) * a.B * a.d + n.chan + v] : 0.f;
  }
  decay_rates<VEC>(a, n, rates, k);

  // c_t = a_t c_{t+1} + a_t dh_t
  float A[T][VEC];
  const int place = waves - 1 - wave;
#pragma unroll
  for (int v = 0; v < VEC; ++v) {
    Map m{1.f, 0.f};
    bool fresh = false;
#pragma unroll
    for (int u = T - 1; u >= 0; --u) {
      float at = decay(k[v], sigmoid_fast(r[u].get(v))).a;
      float g = dh[u].get(v);
      if (f.pad >> u & 1) at = 1.f, g = 0.f;
      if (FLAGS && (f.fresh >> u & 1)) at = 0.f, fresh = true;
      A[u][v] = at;
      m.A *= at;
      m.B = at == 0.f ? 0.f : at * (m.B + g);
    }
    m.A = fresh ? 0.f : fmaxf(m.A, kTiny);
    maps[(place * VEC + v) * 64 + lane] = m;
  }
  __syncthreads();
  float seg_in[VEC], carry[VEC], acc[VEC];
  join_segments<VEC>(c, a, n, rank, waves, maps, win, first, seg_in);
  enter_wave<VEC>(maps, place, seg_in, carry);

#pragma unroll
  for (int v = 0; v < VEC; ++v) acc[v] = 0.f;
  if (n.live && t0 < a.L) {
    // forward again for the states, then back
    float sv[T][VEC], gv[T][VEC], beta[T][VEC], hp[T][VEC];
#pragma unroll
    for (int u = 0; u < T; ++u)
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const float s = sigmoid_fast(r[u].get(v)), g = sigmoid_fast(i[u].get(v));
        const float at = A[u][v];
        float b = __builtin_amdgcn_sqrtf(decay(k[v], s).q);
        if (at == 0.f) b = 1.f;
        float bt = b * g * x[u].get(v);
        if (f.pad >> u & 1) bt = 0.f;
        sv[u][v] = s;
        gv[u][v] = g;
        beta[u][v] = b;
        hp[u][v] = h[v];
        h[v] = apply(Map{at, bt}, h[v]);
      }
#pragma unroll
    for (int u = T - 1; u >= 0; --u) {
      const int t = t0 + u;
      float dx[VEC], dr[VEC], di[VEC];
#pragma unroll
      for (int v = 0; v < VEC; ++v) {
        const bool pad = f.pad >> u & 1;
        const float at = A[u][v], s = sv[u][v], g = gv[u][v];
        const float G = pad ? carry[v] : dh[u].get(v) + carry[v];
        const float gx = g * x[u].get(v), ge = G * beta[u][v] * g;
        float dla = G * at * (hp[u][v] - at * gx * __builtin_amdgcn_rcpf(beta[u][v]));
        // a new document's start depends on no decay, a padded step on nothing
        if (pad || at == 0.f) dla = 0.f;
        const float dls = dla * s;
        acc[v] -= pad || at == 0.f ? 0.f : dls;
        dx[v] = pad ? 0.f : ge;
        di[v] = pad ? 0.f : ge * x[u].get(v) * (1.f - g);
        dr[v] = pad || at == 0.f ? 0.f : -k[v] * dls * (1.f - s);
        carry[v] = at == 0.f ? 0.f : at * G;
      }
      if (t < a.L) {
        Pack<BF16, VEC> o;
        o.put(dx);
        *out_at<BF16, VEC>(a.dx, n, t) = o;
        o.put(dr);
        *out_at<BF16, VEC>(a.dr, n, t) = o;
        o.put(di);
        *out_at<BF16, VEC>(a.di, n, t) = o;
      }
    }
    if (a.dh0 && t0 == 0) {
#pragma unroll
      for (int v = 0; v < VEC; ++v) a.dh0[n.chan + v] = carry[v];
    }
  }
  // the waves' sums in a fixed order
  float* red = reinterpret_cast<float*>(win);
  __syncthreads();
#pragma unroll
  for (int v = 0; v < VEC; ++v) red[(wave * VEC + v) * 64 + lane] = acc[v];
  __syncthreads();
  if (wave == 0 && n.live) {
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
      float s = acc[v];
      for (int w = 1; w < waves; ++w) s += red[(w * VEC + v) * 64 + lane];
      sums[(long long)seg * a.B * a.d + n.chan + v] = s;
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

struct Plan {
  int waves, nseg;
};
Plan plan(int L) {
  Plan p;
  p.waves = L >= kSegment ? kWaves : (L + T - 1) / T;
  p.nseg = (L + kSegment - 1) / kSegment;
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

size_t words_bytes(int L, int B, int d) {
  const Plan p = plan(L);
  return p.nseg == 1 ? 0 : 256 + sizeof(unsigned long long) * (size_t)p.nseg * B * d;
}

hipError_t clear(const Chain& c, const LruArgs& a, hipStream_t st) {
  const long long n = (long long)c.nseg * a.B * a.d;
  const long long blocks = (n + 1023) / 1024;
  timing_before("lru_clear", st);
  hipLaunchKernelGGL(lru_clear_kernel, dim3((unsigned)(blocks < 1024 ? blocks : 1024)), dim3(256),
                     0, st, c.ticket, c.words, n);
  timing_after(st);
  return hipGetLastError();
}

template <bool BF16, int VEC>
hipError_t run(const LruArgs& a, bool grad, hipStream_t st) {
  const Plan p = plan(a.L);
  Chain c{};
  c.nseg = p.nseg;
  c.groups = (int)(((long long)a.B * (a.d / VEC) + 63) / 64);
  char* ws = static_cast<char*>(a.workspace);
  if (p.nseg > 1) {
    c.ticket = reinterpret_cast<unsigned*>(ws);
    c.words = reinterpret_cast<unsigned long long*>(ws + 256);
    if (hipError_t e = clear(c, a, st)) return e;
  }
  const dim3 grid((unsigned)c.groups * p.nseg), block(64 * p.waves);
  const bool flags = a.mask || a.reset;
  if (!grad) {
    timing_before("lru", st);
    if (flags)
      hipLaunchKernelGGL((lru_kernel<BF16, VEC, true>), grid, block, 0, st, a, c);
    else
      hipLaunchKernelGGL((lru_kernel<BF16, VEC, false>), grid, block, 0, st, a, c);
    timing_after(st);
    return hipGetLastError();
  }
  float* sums = reinterpret_cast<float*>(ws + words_bytes(a.L, a.B, a.d));
  timing_before("lru_grad", st);
  if (flags)
    hipLaunchKernelGGL((lru_grad_kernel<BF16, VEC, true>), grid, block, 0, st, a, c, sums);
  else
    hipLaunchKernelGGL((lru_grad_kernel<BF16, VEC, false>), grid, block, 0, st, a, c, sums);
  timing_after(st);
  if (hipError_t e = hipGetLastError()) return e;
  timing_before("lru_sums", st);
  hipLaunchKernelGGL(lru_sums_kernel, dim3((a.d + 63) / 64), dim3(1024), 0, st, a, sums,
                     (long long)p.nseg * a.B);
  timing_after(st);
  return hipGetLastError();
}

hipError_t dispatch(const LruArgs& a, bool grad, bool pairs, hipStream_t st) {
  if (a.bf16) return pairs ? run<true, 2>(a, grad, st) : run<true, 1>(a, grad, st);
  return pairs ? run<false, 2>(a, grad, st) : run<false, 1>(a, grad, st);
}

}  // namespace

size_t lru_workspace_bytes(int L, int B, int d) { return words_bytes(L, B, d); }

size_t lru_grad_workspace_bytes(int L, int B, int d) {
  return words_bytes(L, B, d) + sizeof(float) * (size_t)plan(L).nseg * B * d;
}

long long lru_blocks(int L, int B, int d) {
  return ((long long)B * d + 63) / 64 * plan(L).nseg;  // one channel a lane
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
