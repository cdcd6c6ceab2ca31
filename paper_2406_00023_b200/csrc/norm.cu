// The norm before a block, and the join behind it: the block's output normed, gated, scaled and added to the scaled residual,
// with the next block's norm of the sum; forward and backward.  A row is d values; r(x) = 1 / sqrt(mean x^2 + eps).
//   prenorm  N = x r(x) w
//   join     v = y r(y) w_post (or y w_post),  Xo = a X + b gate v,  N = Xo r(Xo) w_next
// Backward, with xh = Xo r_o, yh = y r_y and <,> the sum over a row:
//   G = dXo + r_o (w_next dN - xh <w_next dN, xh> / d),   dX = a G,   dgate = b <G, w_post yh>
//   u = b gate w_post G,   dY = r_y (u - yh <u, yh> / d),   dw_post = sum_t b gate G yh,   dw_next = sum_t dN xh
// All sums in fp32; a row's norm is taken of the unrounded fp32 sum.
#include "common.cuh"

namespace etr {

struct NormArgs {
  const void *X, *Y, *dXo, *dN, *Xo_in;          // X: input of prenorm, residual of join; Xo_in: the saved sum (backward)
  const float *w_post, *w_next, *gate, *rstd_y, *rstd_o;
  void *Xo, *N, *dX, *dY;
  float *rstd_y_out, *rstd_o_out, *dgate, *part_post, *part_next;
  int T, d, post;
  float eps, a, b;
};

// Sum over a group of TPR threads (a row), in every thread of it.  Two arrays take turns from sum to sum, so that one barrier
// a sum is enough: whoever writes an array again has passed the barrier of the sum between, and so has every reader.
template <int TPR, int BLOCK>
struct RowSum {
  float (*red)[BLOCK / 32];
  int turn;
  __device__ __forceinline__ float operator()(float v) {
    v = warp_sum(v);
    if (TPR <= 32) return v;
    const int warp = threadIdx.x >> 5, first = warp / (TPR / 32) * (TPR / 32);
    if ((threadIdx.x & 31) == 0) red[turn][warp] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < TPR / 32; ++w) v += red[turn][first + w];
    turn ^= 1;
    return v;
  }
};

// A row is held by TPR threads, NV pieces of 16 bytes each: piece u of a thread is piece tg + u TPR of the row.
template <class T> constexpr int PIECE = 16 / (int)sizeof(T);             // values in a piece
template <int TPR> constexpr int NORM_BLOCK = TPR > 256 ? TPR : 256;

template <class T>
__device__ __forceinline__ void unpack(const uint4 q, float* v) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (sizeof(T) == 4) {
      v[i] = __uint_as_float(w[i]);
    } else {
      v[2 * i] = __uint_as_float(w[i] << 16);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}
template <class T>
__device__ __forceinline__ uint4 pack(const float* v) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (sizeof(T) == 4) {
      w[i] = __float_as_uint(v[i]);
    } else {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <int N>
__device__ __forceinline__ void load_gain(const float* w, int col, float* out) {       // w == nullptr: ones
#pragma unroll
  for (int e = 0; e < N; e += 4) {
    const float4 q = w ? *reinterpret_cast<const float4*>(w + col + e) : make_float4(1.f, 1.f, 1.f, 1.f);
    out[e] = q.x; out[e + 1] = q.y; out[e + 2] = q.z; out[e + 3] = q.w;
  }
}

// The rows of up to NT tensors, S tiles ahead.  A thread copies (cp.async) exactly the pieces that it reads itself, so that a
// wait for its own copies is all the synchronisation the ring needs.  S = 0: no ring, read from global memory (rows so
// long that two tiles do not fit).
template <int S, int NT, int BLOCK, int NV>
struct RowRing {
  uint4* smem;
  __device__ __forceinline__ uint4* slot(int stage, int tensor, int u) const { return smem + ((stage * NT + tensor) * NV + u) * BLOCK + threadIdx.x; }
  __device__ __forceinline__ void fetch(int stage, int tensor, int u, const uint4* src) const {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(slot(stage, tensor, u))), "l"(src) : "memory");
  }
  __device__ __forceinline__ void commit() const { asm volatile("cp.async.commit_group;" ::: "memory"); }
  __device__ __forceinline__ void wait() const { asm volatile("cp.async.wait_group %0;" ::"n"(S > 0 ? S - 1 : 0) : "memory"); }
};

// Stages of a ring whose tile takes `bytes`, with `ctas` CTAs of 200 KiB between them on an SM; fewer than two: none.
constexpr int ring_stages(int bytes, int ctas, int most) {
  return 200 * 1024 / ctas / bytes < 2 ? 0 : 200 * 1024 / ctas / bytes < most ? 200 * 1024 / ctas / bytes : most;
}

template <class T, int TPR, int NV, bool JOIN>
struct FwdShape {
  static constexpr int BLOCK = NORM_BLOCK<TPR>, RPB = BLOCK / TPR, NT = JOIN ? 2 : 1;
  static constexpr int CTAS = 768 / BLOCK;
  static constexpr int TILE = NT * BLOCK * NV * 16;
  static constexpr int S = ring_stages(TILE, CTAS, 4), SMEM = S * TILE;
};

// Forward.  JOIN false: prenorm of X.  Blocks walk tiles of RPB rows in strides, with the gains in registers.
template <class T, int TPR, int NV, bool JOIN>
__global__ void __launch_bounds__(NORM_BLOCK<TPR>, FwdShape<T, TPR, NV, JOIN>::CTAS)
norm_fwd_kernel(const NormArgs p) {
  using Sh = FwdShape<T, TPR, NV, JOIN>;
  constexpr int BLOCK = Sh::BLOCK, RPB = Sh::RPB, S = Sh::S, P = PIECE<T>;
  extern __shared__ uint4 ring_smem[];
  __shared__ float red[2][BLOCK / 32];
  RowSum<TPR, BLOCK> row_sum{red, 0};
  const RowRing<S, Sh::NT, BLOCK, NV> ring{ring_smem};
  const int tg = threadIdx.x % TPR, row = threadIdx.x / TPR, np = p.d / P;
  const float inv_d = 1.f / (float)p.d;
  const long long step = (long long)gridDim.x * RPB;
  auto fetch = [&](int stage, long long t) {
    if (t < p.T) {
      const size_t off = (size_t)t * np;
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const int g = tg + u * TPR;
        if (g >= np) continue;
        if (JOIN) ring.fetch(stage, Sh::NT - 1, u, (const uint4*)p.Y + off + g);
        ring.fetch(stage, 0, u, (const uint4*)p.X + off + g);
      }
    }
    ring.commit();
  };
  grid_sync();
  long long t = (long long)blockIdx.x * RPB + row;
  for (int i = 0; i < S - 1; ++i) fetch(i, t + i * step);
  float wp[JOIN ? NV : 1][P], wn[NV][P];
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int g = min(tg + u * TPR, np - 1);
    if (JOIN) load_gain<P>(p.w_post, g * P, wp[u]);
    load_gain<P>(p.N ? p.w_next : nullptr, g * P, wn[u]);
  }
  float gate = p.gate && t < p.T ? p.gate[t] : 1.f;
  int stage = 0;
  for (long long tb = (long long)blockIdx.x * RPB; tb < p.T; tb += step, t += step) {
    const bool live = t < p.T;
    const size_t off = (size_t)(live ? t : 0) * np;
    if (S > 0) {
      fetch(stage == 0 ? S - 1 : stage - 1, t + (S - 1) * step);
      ring.wait();
    }
    auto piece = [&](int tensor, const void* base, int u) {
      const int g = tg + u * TPR;
      if (!live || g >= np) return make_uint4(0, 0, 0, 0);
      return S > 0 ? *ring.slot(stage, tensor, u) : ((const uint4*)base)[off + g];
    };
    float x[NV][P];
#pragma unroll
    for (int u = 0; u < NV; ++u) unpack<T>(piece(0, p.X, u), x[u]);
    if (JOIN) {
      float y[NV][P], f = p.b * gate;
#pragma unroll
      for (int u = 0; u < NV; ++u) unpack<T>(piece(Sh::NT - 1, p.Y, u), y[u]);
      if (p.gate && t + step < p.T) gate = p.gate[t + step];
      if (p.post) {
        float s = 0.f;
#pragma unroll
        for (int u = 0; u < NV; ++u)
#pragma unroll
          for (int e = 0; e < P; ++e) s = fmaf(y[u][e], y[u][e], s);
        const float r = rsqrtf(row_sum(s) * inv_d + p.eps);
        if (p.rstd_y_out && live && tg == 0) p.rstd_y_out[t] = r;
        f *= r;
      }
#pragma unroll
      for (int u = 0; u < NV; ++u) {
#pragma unroll
        for (int e = 0; e < P; ++e) x[u][e] = fmaf(f * y[u][e], wp[u][e], p.a * x[u][e]);
        const int g = tg + u * TPR;
        if (live && g < np) ((uint4*)p.Xo)[off + g] = pack<T>(x[u]);
      }
    }
    if (p.N) {
      float s = 0.f;
#pragma unroll
      for (int u = 0; u < NV; ++u)
#pragma unroll
        for (int e = 0; e < P; ++e) s = fmaf(x[u][e], x[u][e], s);
      const float r = rsqrtf(row_sum(s) * inv_d + p.eps);
      if (p.rstd_o_out && live && tg == 0) p.rstd_o_out[t] = r;
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const int g = tg + u * TPR;
        if (!live || g >= np) continue;
#pragma unroll
        for (int e = 0; e < P; ++e) x[u][e] *= r * wn[u][e];
        ((uint4*)p.N)[off + g] = pack<T>(x[u]);
      }
    }
    stage = S > 0 && stage + 1 < S ? stage + 1 : 0;
  }
}

template <class T, int TPR, int NV, bool JOIN>
struct BwdShape {
  static constexpr int BLOCK = NORM_BLOCK<TPR>, RPB = BLOCK / TPR, NT = JOIN ? 4 : 3;
  static constexpr int CTAS = 512 / BLOCK;
  static constexpr int TILE = NT * BLOCK * NV * 16;
  static constexpr int S = ring_stages(TILE, CTAS, 3), SMEM = S * TILE;
  static constexpr int FOLD = RPB > 1 ? BLOCK * NV * PIECE<T> * 4 : 0;       // one row of partial sums per row group
};

// Backward.  Blocks walk tiles of RPB rows in strides, a thread always on the same columns, so the gains' gradients add up in
// registers; a block leaves one row of partial sums per gain, which norm_dw_kernel adds in order.
// JOIN false: prenorm (Xo_in is its input X, dXo the gradient that comes along the residual, may be NULL; no y).
template <class T, int TPR, int NV, bool JOIN>
__global__ void __launch_bounds__(NORM_BLOCK<TPR>, BwdShape<T, TPR, NV, JOIN>::CTAS)
norm_bwd_kernel(const NormArgs p) {
  using Sh = BwdShape<T, TPR, NV, JOIN>;
  constexpr int BLOCK = Sh::BLOCK, RPB = Sh::RPB, S = Sh::S, P = PIECE<T>;
  extern __shared__ uint4 ring_smem[];
  __shared__ float red[2][BLOCK / 32];
  RowSum<TPR, BLOCK> row_sum{red, 0};
  const RowRing<S, Sh::NT, BLOCK, NV> ring{ring_smem};
  const int tg = threadIdx.x % TPR, row = threadIdx.x / TPR, np = p.d / P;
  const float inv_d = 1.f / (float)p.d;
  const long long step = (long long)gridDim.x * RPB;
  enum { DN, XO, DXO, YY };
  auto fetch = [&](int stage, long long t) {
    if (t < p.T) {
      const size_t off = (size_t)t * np;
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const int g = tg + u * TPR;
        if (g >= np) continue;
        if (p.dN) {
          ring.fetch(stage, DN, u, (const uint4*)p.dN + off + g);
          ring.fetch(stage, XO, u, (const uint4*)p.Xo_in + off + g);
        }
        if (p.dXo) ring.fetch(stage, DXO, u, (const uint4*)p.dXo + off + g);
        if (JOIN) ring.fetch(stage, YY, u, (const uint4*)p.Y + off + g);
      }
    }
    ring.commit();
  };
  grid_sync();
  long long t = (long long)blockIdx.x * RPB + row;
  for (int i = 0; i < S - 1; ++i) fetch(i, t + i * step);
  float wp[JOIN ? NV : 1][P], wn[NV][P], acc_p[JOIN ? NV : 1][P], acc_n[NV][P];
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int g = min(tg + u * TPR, np - 1);
    load_gain<P>(p.dN ? p.w_next : nullptr, g * P, wn[u]);
    if (JOIN) load_gain<P>(p.w_post, g * P, wp[u]);
#pragma unroll
    for (int e = 0; e < P; ++e) {
      acc_n[u][e] = 0.f;
      if (JOIN) acc_p[u][e] = 0.f;
    }
  }
  // a row's scalars are asked for one tile ahead
  float r_o = 0.f, r_y = 1.f, gate = 1.f;
  auto scalars = [&](long long at) {
    if (at >= p.T) return;
    if (p.dN) r_o = p.rstd_o[at];
    if (JOIN && p.post) r_y = p.rstd_y[at];
    if (JOIN && p.gate) gate = p.gate[at];
  };
  scalars(t);
  int stage = 0;
  for (long long tb = (long long)blockIdx.x * RPB; tb < p.T; tb += step, t += step) {
    const bool live = t < p.T;
    const size_t off = (size_t)(live ? t : 0) * np;
    const float ro = r_o, ry = r_y, ga = gate;
    scalars(t + step);
    if (S > 0) {
      fetch(stage == 0 ? S - 1 : stage - 1, t + (S - 1) * step);
      ring.wait();
    }
    auto piece = [&](int tensor, const void* base, int u) {
      const int g = tg + u * TPR;
      if (base == nullptr || !live || g >= np) return make_uint4(0, 0, 0, 0);
      return S > 0 ? *ring.slot(stage, tensor, u) : ((const uint4*)base)[off + g];
    };
    float G[NV][P];
#pragma unroll
    for (int u = 0; u < NV; ++u) unpack<T>(piece(DXO, p.dXo, u), G[u]);
    if (p.dN) {
      float s = 0.f;
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        float dn[P], x[P];
        unpack<T>(piece(DN, p.dN, u), dn);
        unpack<T>(piece(XO, p.Xo_in, u), x);
#pragma unroll
        for (int e = 0; e < P; ++e) {
          const float q = dn[e] * (x[e] * ro);
          acc_n[u][e] += q;
          s = fmaf(q, wn[u][e], s);
        }
      }
      s = row_sum(s) * inv_d;
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        float dn[P], x[P];
        unpack<T>(piece(DN, p.dN, u), dn);
        unpack<T>(piece(XO, p.Xo_in, u), x);
#pragma unroll
        for (int e = 0; e < P; ++e) G[u][e] = fmaf(ro, fmaf(-(x[e] * ro), s, dn[e] * wn[u][e]), G[u][e]);
      }
    }
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int g = tg + u * TPR;
      if (!live || g >= np) continue;
      float out[P];
#pragma unroll
      for (int e = 0; e < P; ++e) out[e] = JOIN ? p.a * G[u][e] : G[u][e];
      ((uint4*)p.dX)[off + g] = pack<T>(out);
    }
    if (JOIN) {
      float s = 0.f;
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        float y[P];
        unpack<T>(piece(YY, p.Y, u), y);
#pragma unroll
        for (int e = 0; e < P; ++e) {
          const float q = p.b * G[u][e] * (y[e] * ry);
          acc_p[u][e] = fmaf(ga, q, acc_p[u][e]);
          s = fmaf(q, wp[u][e], s);
        }
      }
      s = row_sum(s);
      if (p.dgate && live && tg == 0) p.dgate[t] = s;
      const float c = p.post ? s * inv_d : 0.f, f = ga * ry;
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const int g = tg + u * TPR;
        if (!live || g >= np) continue;
        float y[P];
        unpack<T>(piece(YY, p.Y, u), y);
#pragma unroll
        for (int e = 0; e < P; ++e) y[e] = f * fmaf(-(y[e] * ry), c, p.b * G[u][e] * wp[u][e]);
        ((uint4*)p.dY)[off + g] = pack<T>(y);
      }
    }
    stage = S > 0 && stage + 1 < S ? stage + 1 : 0;
  }
  // One row of partial sums per block and gain; where a block has several row groups they are added first, through the
  // ring's memory (every copy into it has arrived: the last groups waited for are empty).
  float* fold = reinterpret_cast<float*>(ring_smem);
#pragma unroll
  for (int which = 0; which < (JOIN ? 2 : 1); ++which) {
    float* part = which ? p.part_post : p.part_next;
    if (part == nullptr) continue;
    if (RPB > 1) __syncthreads();
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int g = tg + u * TPR;
      if (g >= np) continue;
      float* dst = RPB > 1 ? fold + (size_t)row * p.d + g * P : part + (size_t)blockIdx.x * p.d + g * P;
#pragma unroll
      for (int e = 0; e < P; e += 4) {
        const float* v = which ? acc_p[JOIN ? u : 0] : acc_n[u];
        *reinterpret_cast<float4*>(dst + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
      }
    }
    if (RPB > 1) {
      __syncthreads();
      for (int c = threadIdx.x; c < p.d; c += BLOCK) {
        float s = 0.f;
        for (int q = 0; q < RPB; ++q) s += fold[(size_t)q * p.d + c];
        part[(size_t)blockIdx.x * p.d + c] = s;
      }
    }
  }
}

// dw[c] = sum over the blocks' partial rows, in a fixed order; grid y: which weight.
__global__ void __launch_bounds__(256)
norm_dw_kernel(const float* part0, const float* part1, float* __restrict__ dw0, float* __restrict__ dw1, int rows, int d) {
  __shared__ float red[8][33];
  grid_sync();
  const float* part = blockIdx.y ? part1 : part0;
  float* dw = blockIdx.y ? dw1 : dw0;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
  float s = 0.f;
  if (c < d)
    for (int r = warp; r < rows; r += 8) s += part[(size_t)r * d + c];
  red[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < d) {
#pragma unroll
    for (int w = 1; w < 8; ++w) s += red[w][lane];
    dw[c] = s;
  }
}

// ---- launches ----------------------------------------------------------------------------------
static etr_status norm_valid(const etr_norm_config* c) {
  if (c == nullptr) return ETR_ERR_ARG;
  if (c->T < 0 || c->d < 1) return ETR_ERR_ARG;
  if (c->dtype != ETR_F32 && c->dtype != ETR_BF16) return ETR_ERR_ARG;
  if (!(c->eps > 0.f) || !(c->eps < INFINITY) || !(fabsf(c->res_scale) < INFINITY) || !(fabsf(c->branch_scale) < INFINITY)) return ETR_ERR_ARG;
  if (c->d % 8 != 0 || c->d > ETR_NORM_MAX_D) return ETR_ERR_SHAPE;
  return ETR_OK;
}

// need: pointers that have to be there; may: those that can be NULL
static etr_status norm_ptrs(std::initializer_list<const void*> need, std::initializer_list<const void*> may) {
  for (const void* p : need) {
    if (p == nullptr) return ETR_ERR_ARG;
    if (!aligned16(p)) return ETR_ERR_ALIGN;
  }
  for (const void* p : may)
    if (!aligned16(p)) return ETR_ERR_ALIGN;
  return ETR_OK;
}

// Threads per row: as few as hold it with 2 pieces of 16 bytes each, at least a warp, at most 512 (then 4 or 8 pieces).
static int norm_pieces(const NormArgs& p, int dtype) { return p.d * (int)elem_bytes(dtype) / 16; }
static int norm_tpr(int pieces) {
  int tpr = 32;
  while (tpr < 512 && pieces > 2 * tpr) tpr *= 2;
  return tpr;
}

template <template <class, int, int> class K, class T>
static etr_status norm_by_shape(const NormArgs& p, cudaStream_t st) {
  const int pieces = p.d / PIECE<T>, tpr = norm_tpr(pieces);
  switch (tpr) {
    case 32: return pieces <= 32 ? K<T, 32, 1>::run(p, st) : K<T, 32, 2>::run(p, st);
    case 64: return K<T, 64, 2>::run(p, st);
    case 128: return K<T, 128, 2>::run(p, st);
    case 256: return K<T, 256, 2>::run(p, st);
  }
  if (pieces <= 1024) return K<T, 512, 2>::run(p, st);
  if (sizeof(T) == 2 || pieces <= 2048) return K<T, 512, 4>::run(p, st);
  return K<T, 512, sizeof(T) == 2 ? 4 : 8>::run(p, st);
}
template <template <class, int, int> class K>
static etr_status norm_by_type(int dtype, const NormArgs& p, cudaStream_t st) {
  return dtype == ETR_BF16 ? norm_by_shape<K, __nv_bfloat16>(p, st) : norm_by_shape<K, float>(p, st);
}

template <class Sh, class K>
static etr_status norm_launch(const char* name, K kernel, int smem, long long ctas, const NormArgs& p, cudaStream_t st) {
  static std::atomic<unsigned long long> done{0};
  if (smem > 0 && !ensure_dyn_smem(kernel, (size_t)smem, done)) return ETR_ERR_CUDA;
  const long long tiles = ((long long)p.T + Sh::RPB - 1) / Sh::RPB;
  ETR_TIME_BEGIN(name);
  launch_kernel(kernel, (unsigned)(tiles < ctas ? tiles : ctas), Sh::BLOCK, (size_t)smem, st, 1, p);
  ETR_LAUNCH_CHECK();
  return ETR_OK;
}

template <class T, int TPR, int NV>
struct FwdRun {
  template <bool JOIN>
  static etr_status go(const char* name, const NormArgs& p, cudaStream_t st) {
    using Sh = FwdShape<T, TPR, NV, JOIN>;
    return norm_launch<Sh>(name, norm_fwd_kernel<T, TPR, NV, JOIN>, Sh::SMEM, (long long)current_sm_count() * Sh::CTAS, p, st);
  }
  static etr_status run(const NormArgs& p, cudaStream_t st) { return p.Y ? go<true>("join_kernel", p, st) : go<false>("prenorm_kernel", p, st); }
};

// Blocks of the backward kernels: 512 threads on every SM.
static int norm_bwd_blocks(const NormArgs& p, int dtype) {
  const int tpr = norm_tpr(norm_pieces(p, dtype)), block = tpr > 256 ? tpr : 256, rpb = block / tpr;
  const long long want = ((long long)p.T + rpb - 1) / rpb, cap = (long long)current_sm_count() * (512 / block);
  return (int)(want < cap ? want : cap);
}

template <class T, int TPR, int NV>
struct BwdRun {
  template <bool JOIN>
  static etr_status go(const char* name, const NormArgs& p, cudaStream_t st) {
    using Sh = BwdShape<T, TPR, NV, JOIN>;
    return norm_launch<Sh>(name, norm_bwd_kernel<T, TPR, NV, JOIN>, Sh::SMEM > Sh::FOLD ? Sh::SMEM : Sh::FOLD,
                           (long long)current_sm_count() * Sh::CTAS, p, st);
  }
  static etr_status run(const NormArgs& p, cudaStream_t st) { return p.Y ? go<true>("join_bwd_kernel", p, st) : go<false>("prenorm_bwd_kernel", p, st); }
};

static etr_status norm_dw(const etr_norm_config* c, const NormArgs& p, float* dw_next, float* dw_post, cudaStream_t st) {
  if (dw_next == nullptr && dw_post == nullptr) return ETR_OK;
  const bool both = dw_next && dw_post;
  const float* a = dw_next ? p.part_next : p.part_post;
  ETR_TIME_BEGIN("norm_dw_kernel");
  launch_kernel(norm_dw_kernel, dim3(ceil_div(c->d, 32), both ? 2 : 1), 256, 0, st, 1, a, (const float*)p.part_post, dw_next ? dw_next : dw_post,
                dw_post, norm_bwd_blocks(p, c->dtype), c->d);
  ETR_LAUNCH_CHECK();
  return ETR_OK;
}

static NormArgs norm_args(const etr_norm_config* c) {
  NormArgs p = {};
  p.T = c->T; p.d = c->d; p.post = c->post_norm != 0;
  p.eps = c->eps; p.a = c->res_scale; p.b = c->branch_scale;
  return p;
}

}  // namespace etr

using namespace etr;

extern "C" {

etr_status etr_norm_validate(const etr_norm_config* c) { return norm_valid(c); }

etr_status etr_norm_workspace_bytes(const etr_norm_config* c, size_t* bytes) {
  if (bytes == nullptr) return ETR_ERR_ARG;
  ETR_TRY(norm_valid(c));
  *bytes = align_up((size_t)2 * current_sm_count() * 2 * c->d * 4, 256);
  return ETR_OK;
}

etr_status etr_prenorm(const etr_norm_config* c, const void* X, const float* w, void* N, float* rstd, void* stream) {
  ETR_TRY(norm_valid(c));
  if (c->T == 0) return ETR_OK;
  ETR_TRY(norm_ptrs({X, N}, {w, rstd}));
  NormArgs p = norm_args(c);
  p.X = X; p.w_next = w; p.N = N; p.rstd_o_out = rstd;
  return norm_by_type<FwdRun>(c->dtype, p, (cudaStream_t)stream);
}

etr_status etr_join(const etr_norm_config* c, const void* X, const void* Y, const float* w_post, const float* gate, const float* w_next,
                    void* Xo, void* N, float* rstd_y, float* rstd_o, void* stream) {
  ETR_TRY(norm_valid(c));
  if (c->T == 0) return ETR_OK;
  ETR_TRY(norm_ptrs({X, Y, Xo}, {w_post, gate, w_next, N, rstd_y, rstd_o}));
  NormArgs p = norm_args(c);
  p.X = X; p.Y = Y; p.w_post = w_post; p.gate = gate; p.w_next = w_next; p.Xo = Xo; p.N = N;
  p.rstd_y_out = rstd_y; p.rstd_o_out = rstd_o;
  return norm_by_type<FwdRun>(c->dtype, p, (cudaStream_t)stream);
}

etr_status etr_prenorm_bwd(const etr_norm_config* c, const void* dN, const void* X, const float* w, const float* rstd, const void* dres,
                           void* dX, float* dw, void* ws, void* stream) {
  ETR_TRY(norm_valid(c));
  ETR_TRY(norm_ptrs({}, {dN, X, w, rstd, dres, dX, dw, ws}));
  if (c->T > 0) ETR_TRY(norm_ptrs({dN, X, rstd, dX}, {}));
  if (dw) ETR_TRY(norm_ptrs({ws}, {}));
  NormArgs p = norm_args(c);
  p.dN = dN; p.Xo_in = X; p.w_next = w; p.rstd_o = rstd; p.dXo = dres; p.dX = dX;
  p.part_next = dw ? (float*)ws : nullptr;
  if (c->T > 0) ETR_TRY(norm_by_type<BwdRun>(c->dtype, p, (cudaStream_t)stream));
  return norm_dw(c, p, dw, nullptr, (cudaStream_t)stream);
}

etr_status etr_join_bwd(const etr_norm_config* c, const void* dXo, const void* dN, const void* Y, const void* Xo, const float* w_post,
                        const float* gate, const float* w_next, const float* rstd_y, const float* rstd_o, void* dX, void* dY,
                        float* dw_post, float* dgate, float* dw_next, void* ws, void* stream) {
  ETR_TRY(norm_valid(c));
  ETR_TRY(norm_ptrs({}, {dXo, dN, Y, Xo, w_post, gate, w_next, rstd_y, rstd_o, dX, dY, dw_post, dgate, dw_next, ws}));
  if (c->T > 0) {
    ETR_TRY(norm_ptrs({Y, dX, dY}, {}));
    if (dXo == nullptr && dN == nullptr) return ETR_ERR_ARG;
    if (dN) ETR_TRY(norm_ptrs({Xo, rstd_o}, {}));
    if (c->post_norm) ETR_TRY(norm_ptrs({rstd_y}, {}));
  }
  if (dw_next && dN == nullptr && c->T > 0) return ETR_ERR_ARG;
  if (dw_post || dw_next) ETR_TRY(norm_ptrs({ws}, {}));
  NormArgs p = norm_args(c);
  p.dXo = dXo; p.dN = dN; p.Y = Y; p.Xo_in = Xo; p.w_post = w_post; p.gate = gate; p.w_next = w_next; p.rstd_y = rstd_y; p.rstd_o = rstd_o;
  p.dX = dX; p.dY = dY; p.dgate = dgate;
  p.part_next = dw_next ? (float*)ws : nullptr;
  p.part_post = dw_post ? (float*)ws + (size_t)current_sm_count() * 2 * c->d : nullptr;
  if (c->T > 0) ETR_TRY(norm_by_type<BwdRun>(c->dtype, p, (cudaStream_t)stream));
  return norm_dw(c, p, dw_next, dw_post, (cudaStream_t)stream);
}

}  // extern "C"
