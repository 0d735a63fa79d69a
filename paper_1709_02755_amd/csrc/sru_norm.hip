// Between two blocks of a residual network: the norm of the block's output,
// its gate, the residual scale and sum, and the norm before the next block,
//   n = y rstd(y) w_post,  u = n gate(z),  x' = x + scale u,  o = x' rstd(x') w_pre
// with rstd(v) = 1 / sqrt(mean(v^2) + eps), and its gradient.
//
// Both are bound by memory: a row's tensors are read once into registers, all
// in 16-byte loads (but see by_width), its sums are taken there, and the
// results leave rounded once.  The gradient works x' out again from x, y and z
// rather than reading x_out, so that no rounded value enters it.  16384 x 1024,
// bf16 beside an fp32 residual, each call repeated by itself: 50 us for 235 MB (4.7
// TB/s) and 88 us for 369 MB (4.2 TB/s); in turn, as in training, the kernels take 49
// and 76 + 5, the gradient's with part of its inputs still in the caches.  8 x 1024
// bf16: 4.4 us, a launch.
#include <type_traits>

#include "sru_device.h"
#include "sru_lanes.h"
#include "sru_lm.h"

namespace sru {
namespace {

// 16 bytes in memory, and where an element may lie rather than on 16 bytes.
typedef unsigned Quad __attribute__((ext_vector_type(4)));
template <bool BF16>
struct Mem {
  using T = float;
  typedef Quad Loose __attribute__((aligned(4)));
};
template <>
struct Mem<true> {
  using T = uint16_t;
  typedef Quad Loose __attribute__((aligned(2)));
};

// VE consecutive elements to and from floats; 16-byte accesses (two for 8
// fp32 values) unless VE is 1.  TAIL: anywhere, and only the first `left` of them
// may be there; the others are 0.
template <bool BF16, int VE, bool TAIL>
__device__ __forceinline__ void load(const typename Mem<BF16>::T* p, int left, float* f) {
  constexpr int E = BF16 ? 8 : 4;  // of 16 bytes
  if constexpr (TAIL) {
    static_assert(VE % E == 0, "16 bytes");
    if (left >= VE) {
#pragma unroll
      for (int i = 0; i < VE; i += E) {
        const Quad q = *reinterpret_cast<const typename Mem<BF16>::Loose*>(p + i);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          if constexpr (BF16) {
            f[2 * w] = __uint_as_float(q[w] << 16);
            f[2 * w + 1] = __uint_as_float(q[w] & 0xffff0000u);
          } else {
            f[i + w] = __uint_as_float(q[w]);
          }
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        f[i] = 0.f;
        if (i < left) load<BF16, 1, false>(p + i, 1, f + i);
      }
    }
  } else if constexpr (VE == 1) {
    if constexpr (BF16) f[0] = __uint_as_float((unsigned)*p << 16);
    else f[0] = *p;
  } else if constexpr (BF16) {
    static_assert(VE == 8, "16 bytes");
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const unsigned w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int i = 0; i < VE; i += 4) {
      const float4 v = *reinterpret_cast<const float4*>(p + i);
      f[i] = v.x;
      f[i + 1] = v.y;
      f[i + 2] = v.z;
      f[i + 3] = v.w;
    }
  }
}
// LAST: past the caches, for what is not read again soon.
template <bool BF16, int VE, bool TAIL, bool LAST>
__device__ __forceinline__ void store(typename Mem<BF16>::T* p, int left, const float* f) {
  using Q = std::conditional_t<TAIL, typename Mem<BF16>::Loose, Quad>;
  if (TAIL && left < VE) {
#pragma unroll
    for (int i = 0; i < VE; ++i)
      if (i < left) store<BF16, 1, false, false>(p + i, 1, f + i);
  } else if constexpr (VE == 1) {
    if constexpr (BF16) *p = __builtin_bit_cast(uint16_t, (__bf16)f[0]);
    else *p = f[0];
  } else if constexpr (BF16) {
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = (unsigned)__builtin_bit_cast(uint16_t, (__bf16)f[2 * i]) |
             ((unsigned)__builtin_bit_cast(uint16_t, (__bf16)f[2 * i + 1]) << 16);
    const Quad q = {w[0], w[1], w[2], w[3]};
    if constexpr (LAST) __builtin_nontemporal_store(q, reinterpret_cast<Q*>(p));
    else *reinterpret_cast<Q*>(p) = q;
  } else {
#pragma unroll
    for (int i = 0; i < VE; i += 4) {
      const Quad q = {__float_as_uint(f[i]), __float_as_uint(f[i + 1]), __float_as_uint(f[i + 2]),
                      __float_as_uint(f[i + 3])};
      if constexpr (LAST) __builtin_nontemporal_store(q, reinterpret_cast<Q*>(p + i));
      else *reinterpret_cast<Q*>(p + i) = q;
    }
  }
}

// How a kernel holds a row: LANES threads, each C chunks of VE consecutive
// columns, the chunks of a row dealt to its threads in turn.  Rows of up to a
// wave (16, 32 or 64 lanes) come 256 / LANES to a workgroup; their sums need no
// barrier.
// TAIL: a row may start between 16-byte boundaries and end inside a chunk.
template <int VE_, int C_, int LANES_, bool TAIL_ = false>
struct Hold {
  static constexpr int VE = VE_, C = C_, LANES = LANES_, F = VE_ * C_;
  static constexpr bool TAIL = TAIL_;
  static constexpr int NW = LANES_ <= 64 ? 1 : LANES_ / 64;  // waves of a row
  static constexpr int ROWS = NW == 1 ? 256 / LANES_ : 1;
  static constexpr int THREADS = LANES_ * ROWS;
  __device__ static int lane() { return NW == 1 ? threadIdx.x % LANES : threadIdx.x; }
  __device__ static int sub() { return NW == 1 ? threadIdx.x / LANES : 0; }
  __device__ static int col(int c) { return (c * LANES + lane()) * VE; }
};

// F columns of a row as they lie in memory; columns past d are 0.
template <class H, bool BF16>
struct Raw {
  static_assert(!H::TAIL, "rows of whole pieces, or one by one");
  static constexpr int Q = H::VE * (BF16 ? 2 : 4) / 16;  // 16-byte pieces of a chunk
  uint4 q[Q ? H::C * Q : 1];
  typename Mem<BF16>::T e[Q ? 1 : H::C];
  __device__ __forceinline__ void load(const void* p, long long off, int d) {
    const auto* at = static_cast<const typename Mem<BF16>::T*>(p) + off;
#pragma unroll
    for (int c = 0; c < H::C; ++c) {
      const int col = H::col(c);
      if constexpr (Q > 0) {
#pragma unroll
        for (int i = 0; i < Q; ++i) {
          q[c * Q + i] = make_uint4(0, 0, 0, 0);
          if (col < d) q[c * Q + i] = reinterpret_cast<const uint4*>(at + col)[i];
        }
      } else {
        e[c] = 0;
        if (col < d) e[c] = at[col];
      }
    }
  }
  __device__ __forceinline__ void get(float (&f)[H::F]) const {
#pragma unroll
    for (int c = 0; c < H::C; ++c) {
      if constexpr (Q > 0 && BF16) {
        const unsigned w[4] = {q[c].x, q[c].y, q[c].z, q[c].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          f[c * H::VE + 2 * i] = __uint_as_float(w[i] << 16);
          f[c * H::VE + 2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
      } else if constexpr (Q > 0) {
#pragma unroll
        for (int i = 0; i < Q; ++i) {
          const uint4& u = q[c * Q + i];
          f[c * H::VE + 4 * i] = __uint_as_float(u.x);
          f[c * H::VE + 4 * i + 1] = __uint_as_float(u.y);
          f[c * H::VE + 4 * i + 2] = __uint_as_float(u.z);
          f[c * H::VE + 4 * i + 3] = __uint_as_float(u.w);
        }
      } else if constexpr (BF16) {
        f[c] = __uint_as_float((unsigned)e[c] << 16);
      } else {
        f[c] = e[c];
      }
    }
  }
};

// F columns of a row; columns past d are 0.
template <class H, bool BF16>
__device__ __forceinline__ void load_row(const void* p, long long off, int d, float (&f)[H::F]) {
  const auto* q = static_cast<const typename Mem<BF16>::T*>(p) + off;
#pragma unroll
  for (int c = 0; c < H::C; ++c) {
    const int col = H::col(c);
    if (col < d) {
      load<BF16, H::VE, H::TAIL>(q + col, d - col, f + c * H::VE);
    } else {
#pragma unroll
      for (int j = 0; j < H::VE; ++j) f[c * H::VE + j] = 0.f;
    }
  }
}
template <class H, bool BF16, bool LAST = false>
__device__ __forceinline__ void store_row(const void* p, long long off, int d,
                                          const float (&f)[H::F]) {
  auto* q = static_cast<typename Mem<BF16>::T*>(const_cast<void*>(p)) + off;
#pragma unroll
  for (int c = 0; c < H::C; ++c) {
    const int col = H::col(c);
    if (col < d) store<BF16, H::VE, H::TAIL, LAST>(q + col, d - col, f + c * H::VE);
  }
}

// The sum over a row's threads, in each of them, always in the same order.
template <class H>
__device__ __forceinline__ float row_sum(float v, float* lds) {
  v = lanes_sum<(H::LANES < 64 ? H::LANES : 64)>(v);
  if constexpr (H::NW > 1) {
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = lds[0];
#pragma unroll
    for (int w = 1; w < H::NW; ++w) v += lds[w];
    __syncthreads();
  }
  return v;
}

__device__ __forceinline__ float rstd_of(float sum, int d, float eps) {
  return 1.f / sqrtf(sum / (float)d + eps);
}

template <class H, bool ABF, bool RBF>
__global__ __launch_bounds__(H::THREADS) void norm_kernel(NormArgs a) {
  __shared__ float lds[H::NW];
  const int d = a.d;
  for (long long m0 = (long long)blockIdx.x * H::ROWS; m0 < a.M;
       m0 += (long long)gridDim.x * H::ROWS) {
    const long long m = m0 + H::sub();
    if (H::NW == 1 && m >= a.M) break;  // the threads of a row meet no barrier
    float x[H::F], rx = 0.f, ry = 0.f;
    load_row<H, RBF>(a.x.p, m * a.x.ld, d, x);
    if (a.y.p) {
      float y[H::F], z[H::F], w[H::F];
      load_row<H, ABF>(a.y.p, m * a.y.ld, d, y);
      if (a.z.p) load_row<H, ABF>(a.z.p, m * a.z.ld, d, z);
      if (a.w_post) {
        load_row<H, false>(a.w_post, 0, d, w);
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < H::F; ++j) s = fmaf(y[j], y[j], s);
        ry = rstd_of(row_sum<H>(s, lds), d, a.eps);
#pragma unroll
        for (int j = 0; j < H::F; ++j) y[j] = y[j] * ry * w[j];
      }
      if (a.z.p) {
#pragma unroll
        for (int j = 0; j < H::F; ++j) {
          const float sg = sigmoid_fast(z[j]);
          y[j] *= a.silu ? z[j] * sg : sg;
        }
      }
      if (a.scale) load_row<H, false>(a.scale, 0, d, w);
#pragma unroll
      for (int j = 0; j < H::F; ++j) x[j] = a.scale ? fmaf(w[j], y[j], x[j]) : x[j] + y[j];
      // next read a block later (16384 x 1024 bf16 beside fp32 56 -> 51 us)
      store_row<H, RBF, true>(a.x_out.p, m * a.x_out.ld, d, x);
    }
    if (a.w_pre) {
      float w[H::F];
      load_row<H, false>(a.w_pre, 0, d, w);
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < H::F; ++j) s = fmaf(x[j], x[j], s);
      rx = rstd_of(row_sum<H>(s, lds), d, a.eps);
#pragma unroll
      for (int j = 0; j < H::F; ++j) w[j] *= x[j] * rx;
      store_row<H, ABF>(a.o.p, m * a.o.ld, d, w);
    }
    if (H::lane() == 0) {
      a.rstd[2 * m] = ry;
      a.rstd[2 * m + 1] = rx;
    }
  }
}

// t = do w_pre, xh = x' rstd_x:  dx = dx_out + rstd_x (t - xh mean(t xh));
// du = dx scale, dz = du n gate'(z), dn = du gate(z);
// t = dn w_post, yh = y rstd_y:  dy = rstd_y (t - yh mean(t yh)).
// Every workgroup adds its rows' terms of the three parameter gradients in
// registers and leaves one row of sums, [workgroup, 3, d].
template <class H, bool ABF, bool RBF>
struct GradRow {
  Raw<H, RBF> x, dx;
  Raw<H, ABF> y, z, go;
  __device__ __forceinline__ void load(const NormArgs& a, long long m) {
    if (m >= a.M) return;
    x.load(a.x.p, m * a.x.ld, a.d);
    if (a.y.p) y.load(a.y.p, m * a.y.ld, a.d);
    if (a.z.p) z.load(a.z.p, m * a.z.ld, a.d);
    if (a.go.p) go.load(a.go.p, m * a.go.ld, a.d);
    if (a.dx_out.p) dx.load(a.dx_out.p, m * a.dx_out.ld, a.d);
  }
};

// When a row's tensors are loaded.  Rows of up to a wave: all at once, in front
// (2 or 3 waves run on a SIMD then, fewer than with loads where they are used,
// but with more in flight: 16384 x 1024 bf16 beside fp32 104 -> 91 us, 65536 x
// 256 145 -> 85; left to itself, the compiler takes registers past what 2 waves
// can have, and 1 takes 109 us).  256 threads to a row, which wait for each other twice a row:
// while the row before is worked on (8192 x 2048 121 -> 97 us).  Wider rows: each
// where it is used (4096 x 4096 98 us, 105 in front).
template <class H, bool ABF, bool RBF>
__global__ __launch_bounds__(H::THREADS, H::LANES > 256 ? 1 : H::F == 16 ? 2 : 3) void
norm_grad_kernel(NormArgs a) {
  constexpr bool AHEAD = H::LANES == 256, WHOLE = AHEAD || H::NW == 1;
  __shared__ float lds[H::NW];
  __shared__ float sums[H::ROWS > 1 ? H::THREADS * H::F : 1];
  const int d = a.d;
  float gw_post[H::F], gscale[H::F], gw_pre[H::F];
#pragma unroll
  for (int j = 0; j < H::F; ++j) gw_post[j] = gscale[j] = gw_pre[j] = 0.f;

  const long long step = (long long)gridDim.x * H::ROWS;
  struct None {};
  std::conditional_t<WHOLE, GradRow<H, ABF, RBF>, None> row, next;
  if constexpr (AHEAD) next.load(a, (long long)blockIdx.x * H::ROWS + H::sub());
  for (long long m0 = (long long)blockIdx.x * H::ROWS; m0 < a.M; m0 += step) {
    const long long m = m0 + H::sub();
    if (H::NW == 1 && m >= a.M) break;
    if constexpr (AHEAD) {
      row = next;
      next.load(a, m + step);
    } else if constexpr (WHOLE) {
      row.load(a, m);
    }
    float x[H::F], y[H::F], z[H::F], u[H::F], dx[H::F], w[H::F];
    if constexpr (WHOLE) {
      row.x.get(x);
      if (a.y.p) row.y.get(y);
      if (a.z.p) row.z.get(z);
      if (a.dx_out.p) row.dx.get(dx);
    } else {
      load_row<H, RBF>(a.x.p, m * a.x.ld, d, x);
      if (a.y.p) load_row<H, ABF>(a.y.p, m * a.y.ld, d, y);
      if (a.z.p) load_row<H, ABF>(a.z.p, m * a.z.ld, d, z);
      if (a.dx_out.p) load_row<H, RBF>(a.dx_out.p, m * a.dx_out.ld, d, dx);
    }
    if (!a.dx_out.p) {
#pragma unroll
      for (int j = 0; j < H::F; ++j) dx[j] = 0.f;
    }
    const float ry = a.w_post ? a.rstd[2 * m] : 1.f;
    // y becomes yh; u = n gate(z)
    if (a.y.p) {
#pragma unroll
      for (int j = 0; j < H::F; ++j) u[j] = y[j] *= ry;
      if (a.w_post) {
        load_row<H, false>(a.w_post, 0, d, w);
#pragma unroll
        for (int j = 0; j < H::F; ++j) u[j] *= w[j];
      }
      if (a.z.p) {
#pragma unroll
        for (int j = 0; j < H::F; ++j) {
          const float sg = sigmoid_fast(z[j]);
          u[j] *= a.silu ? z[j] * sg : sg;
        }
      }
      if (a.scale) load_row<H, false>(a.scale, 0, d, w);
#pragma unroll
      for (int j = 0; j < H::F; ++j) x[j] = a.scale ? fmaf(w[j], u[j], x[j]) : x[j] + u[j];
    }
    if (a.w_pre && a.go.p) {
      const float rx = a.rstd[2 * m + 1];
      float t[H::F];
      if constexpr (WHOLE) row.go.get(t);
      else load_row<H, ABF>(a.go.p, m * a.go.ld, d, t);
      load_row<H, false>(a.w_pre, 0, d, w);
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < H::F; ++j) {
        x[j] *= rx;
        gw_pre[j] = fmaf(t[j], x[j], gw_pre[j]);
        t[j] *= w[j];
        s = fmaf(t[j], x[j], s);
      }
      s = row_sum<H>(s, lds) / (float)d;
#pragma unroll
      for (int j = 0; j < H::F; ++j) dx[j] += rx * (t[j] - x[j] * s);
    }
    store_row<H, RBF, true>(a.dx.p, m * a.dx.ld, d, dx);
    if (!a.y.p) continue;
#pragma unroll
    for (int j = 0; j < H::F; ++j) gscale[j] = fmaf(dx[j], u[j], gscale[j]);
    // dx becomes du
    if (a.scale) {
      load_row<H, false>(a.scale, 0, d, w);
#pragma unroll
      for (int j = 0; j < H::F; ++j) dx[j] *= w[j];
    }
    if (a.w_post) {
      load_row<H, false>(a.w_post, 0, d, w);
    } else {
#pragma unroll
      for (int j = 0; j < H::F; ++j) w[j] = 1.f;
    }
    // z becomes dz, dx becomes dn
    if (a.z.p) {
#pragma unroll
      for (int j = 0; j < H::F; ++j) {
        const float sg = sigmoid_fast(z[j]);
        const float gate = a.silu ? z[j] * sg : sg;
        const float slope = a.silu ? fmaf(gate, 1.f - sg, sg) : sg * (1.f - sg);
        z[j] = dx[j] * (y[j] * w[j]) * slope;
        dx[j] *= gate;
      }
      store_row<H, ABF>(a.dz.p, m * a.dz.ld, d, z);
    }
    if (a.w_post) {
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < H::F; ++j) {
        gw_post[j] = fmaf(dx[j], y[j], gw_post[j]);
        dx[j] *= w[j];
        s = fmaf(dx[j], y[j], s);
      }
      s = row_sum<H>(s, lds) / (float)d;
#pragma unroll
      for (int j = 0; j < H::F; ++j) dx[j] = ry * (dx[j] - y[j] * s);
    }
    store_row<H, ABF>(a.dy.p, m * a.dy.ld, d, dx);
  }

  // the workgroup's sums, its rows' waves added in order
  float* const out = a.partial + (long long)blockIdx.x * 3 * d;
  auto leave = [&](float(&g)[H::F], int q) {
    if constexpr (H::ROWS > 1) {
      __syncthreads();
#pragma unroll
      for (int j = 0; j < H::F; ++j) sums[(H::sub() * H::F + j) * H::LANES + H::lane()] = g[j];
      __syncthreads();
      if (H::sub() != 0) return;
#pragma unroll
      for (int j = 0; j < H::F; ++j) {
        float s = g[j];
#pragma unroll
        for (int r = 1; r < H::ROWS; ++r) s += sums[(r * H::F + j) * H::LANES + H::lane()];
        g[j] = s;
      }
    }
    store_row<H, false>(out, (long long)q * d, d, g);
  };
  if (a.dw_post) leave(gw_post, 0);
  if (a.dscale) leave(gscale, 1);
  if (a.dw_pre) leave(gw_pre, 2);
}

// Column sums of [rows, 3, d]: 64 columns a workgroup, its 16 waves take every
// 16th row and meet in a fixed order.
__global__ __launch_bounds__(1024) void norm_sums_kernel(NormArgs a, int rows) {
  __shared__ float red[16 * 64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int groups = (a.d + 63) / 64;
  const int q = blockIdx.x / groups, col = (blockIdx.x - q * groups) * 64 + lane;
  float* const out = q == 0 ? a.dw_post : q == 1 ? a.dscale : a.dw_pre;
  if (!out) return;  // the whole workgroup
  float s = 0.f;
  if (col < a.d) {
    const float* p = a.partial + (long long)q * a.d + col;
    const long long stride = 3LL * a.d;
#pragma unroll 8
    for (int r = w; r < rows; r += 16) s += p[r * stride];
  }
  red[w * 64 + lane] = s;
  __syncthreads();
  if (w == 0 && col < a.d) {
#pragma unroll
    for (int i = 1; i < 16; ++i) s += red[i * 64 + lane];
    out[col] = s;
  }
}

// Workgroups of the gradient: each leaves one row of sums, so only as many as
// run at a time (by the registers they take; 8192 x 2048 with 512 of them 105 us, 96).
int rows_at_once(int d) { return d <= 128 ? 16 : d <= 256 ? 8 : d <= 1024 ? 4 : 1; }
int grad_blocks(int M, int d) {
  const int most = d <= 512 || (d > 1024 && d <= 2048) ? 768 : d <= 4096 ? 512 : 256;
  const int want = (int)(((long long)M + rows_at_once(d) - 1) / rows_at_once(d));
  return want < most ? want : most;
}

// H: a row's threads and columns in the forward, G: in the gradient.
template <bool ABF, bool RBF, class H, class G = H>
hipError_t launch(const NormArgs& a, bool grad, hipStream_t st) {
  if (grad) {
    static_assert(G::F == 8 || G::F == 16, "columns of a thread");
    const int blocks = grad_blocks(a.M, a.d);
    timing_before("norm_grad", st);
    hipLaunchKernelGGL((norm_grad_kernel<G, ABF, RBF>), dim3(blocks), dim3(G::THREADS), 0, st, a);
    timing_after(st);
    if (hipError_t e = hipGetLastError()) return e;
    if (!a.dw_post && !a.dscale && !a.dw_pre) return hipSuccess;
    timing_before("norm_sums", st);
    hipLaunchKernelGGL(norm_sums_kernel, dim3(3 * ((a.d + 63) / 64)), dim3(1024), 0, st, a,
                       blocks);
    timing_after(st);
    return hipGetLastError();
  }
  const long long want = ((long long)a.M + H::ROWS - 1) / H::ROWS;
  timing_before("norm", st);
  hipLaunchKernelGGL((norm_kernel<H, ABF, RBF>),
                     dim3((unsigned)(want < kMaxGrid ? want : kMaxGrid)), dim3(H::THREADS), 0, st,
                     a);
  timing_after(st);
  return hipGetLastError();
}

// Threads a row and columns a thread by the width: a row's columns stay in
// registers, 8 to a thread (16 up to 1024 columns, where one wave then holds a
// row and needs no barrier, and past 8192; past 4096 in the forward, which has
// registers to spare and waits for fewer waves then: 2000 x 6000 fp32 60 -> 50 us,
// while the gradient takes 97 with 8 and 103 with 16).
// Rows that are not whole pieces of 16 bytes take them all the same (TAIL: 16384 x
// 1001 bf16 beside fp32, forward 93 -> 53 us; 2000 x 6001 fp32, gradient 146 -> 96),
// but for the gradient up to 2048 columns, which takes elements one by one (10154 x
// 1277 bf16 92 us and 166 so, 5123 x 301 fp32 22 and 24: pieces that lie on odd
// elements are slow to store).
template <int VE, bool ABF, bool RBF, bool TAIL>
hipError_t by_width(const NormArgs& a, bool grad, hipStream_t st) {
  constexpr int C = 8 / VE, G = TAIL ? 1 : VE, D = 8 / G;
  if (a.d <= 128)
    return launch<ABF, RBF, Hold<VE, C, 16, TAIL>, Hold<G, D, 16>>(a, grad, st);
  if (a.d <= 256)
    return launch<ABF, RBF, Hold<VE, C, 32, TAIL>, Hold<G, D, 32>>(a, grad, st);
  if (a.d <= 512)
    return launch<ABF, RBF, Hold<VE, C, 64, TAIL>, Hold<G, D, 64>>(a, grad, st);
  if (a.d <= 1024)
    return launch<ABF, RBF, Hold<VE, 2 * C, 64, TAIL>, Hold<G, 2 * D, 64>>(a, grad, st);
  if (a.d <= 2048)
    return launch<ABF, RBF, Hold<VE, C, 256, TAIL>, Hold<G, D, 256>>(a, grad, st);
  if (a.d <= 4096) return launch<ABF, RBF, Hold<VE, C, 512, TAIL>>(a, grad, st);
  if (a.d <= 8192)
    return launch<ABF, RBF, Hold<VE, 2 * C, 512, TAIL>, Hold<VE, C, 1024, TAIL>>(a, grad, st);
  return launch<ABF, RBF, Hold<VE, 2 * C, 1024, TAIL>>(a, grad, st);
}

// Whether every row of every tensor is whole pieces of 16 bytes.
bool whole_pieces(const NormArgs& a) {
  const int ve = a.act_bf16 ? 8 : 4;
  if (a.d % ve) return false;
  auto rows = [](const Rows& r, bool bf16) {
    return !r.p || ((reinterpret_cast<uintptr_t>(r.p) | (uintptr_t)(r.ld * (bf16 ? 2 : 4))) & 15) == 0;
  };
  auto vec = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; };
  const bool A = a.act_bf16, R = a.res_bf16;
  return rows(a.x, R) && rows(a.y, A) && rows(a.z, A) && rows(a.x_out, R) && rows(a.o, A) &&
         rows(a.dx_out, R) && rows(a.go, A) && rows(a.dx, R) && rows(a.dy, A) && rows(a.dz, A) &&
         vec(a.w_post) && vec(a.scale) && vec(a.w_pre);
}

template <int VE, bool ABF, bool RBF>
hipError_t by_pieces(const NormArgs& a, bool grad, hipStream_t st) {
  return whole_pieces(a) ? by_width<VE, ABF, RBF, false>(a, grad, st)
                         : by_width<VE, ABF, RBF, true>(a, grad, st);
}

hipError_t dispatch(const NormArgs& a, bool grad, hipStream_t st) {
  if (!a.act_bf16) return by_pieces<4, false, false>(a, grad, st);
  if (!a.res_bf16) return by_pieces<8, true, false>(a, grad, st);
  return by_pieces<8, true, true>(a, grad, st);
}

}  // namespace

hipError_t norm_launch(const NormArgs& a, hipStream_t stream) { return dispatch(a, false, stream); }

size_t norm_grad_workspace_bytes(int M, int d) {
  return sizeof(float) * 3 * (size_t)d * grad_blocks(M, d);
}

hipError_t norm_grad_launch(const NormArgs& a, hipStream_t stream) {
  return dispatch(a, true, stream);
}

}  // namespace sru
