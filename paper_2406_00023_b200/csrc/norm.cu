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

// How rows lie on a block's threads: tpr threads hold a row (a power of two up to 32, or whole warps), NV pieces of 16 bytes each
// (piece u of a thread is piece tg + u tpr of the row), rpb rows side by side in a block.
struct RowShape { int tpr, rpb, stages; };

// Sum over a row's threads, in every one of them.  Two arrays take turns from sum to sum, so that one barrier a sum is
// enough: whoever writes an array again has passed the barrier of the sum between, and so has every reader.
constexpr int NORM_MAX_WARPS = 16;                // 512 threads
struct RowSum {
  float (*red)[NORM_MAX_WARPS];                   // [2][NORM_MAX_WARPS]
  int tpr, turn;
  __device__ __forceinline__ float operator()(float v) {
    if (tpr <= 32) {
      for (int o = tpr >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
      return v;
    }
    v = warp_sum(v);
    const int warp = threadIdx.x >> 5, wpr = tpr >> 5, first = warp / wpr * wpr;
    if ((threadIdx.x & 31) == 0) red[turn][warp] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll 4
    for (int w = 0; w < wpr; ++w) v += red[turn][first + w];
    turn ^= 1;
    return v;
  }
};

template <int N>
__device__ __forceinline__ void load_gain(const float* w, int col, float* out) {       // w == nullptr: ones
#pragma unroll
  for (int e = 0; e < N; e += 4) {
    const float4 q = w ? *reinterpret_cast<const float4*>(w + col + e) : make_float4(1.f, 1.f, 1.f, 1.f);
    out[e] = q.x; out[e + 1] = q.y; out[e + 2] = q.z; out[e + 3] = q.w;
  }
}

// The rows of up to NT tensors, tiles ahead of their use.  A thread copies (cp.async) exactly the pieces that it reads
// itself, so that a wait for its own copies is all the synchronisation the ring needs.
template <int NT, int NV>
struct RowRing {
  uint4* smem;
  __device__ __forceinline__ uint4* slot(int stage, int tensor, int u) const { return smem + ((stage * NT + tensor) * NV + u) * blockDim.x + threadIdx.x; }
  __device__ __forceinline__ void fetch(int stage, int tensor, int u, const uint4* src) const {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(slot(stage, tensor, u))), "l"(src) : "memory");
  }
  __device__ __forceinline__ void commit() const { asm volatile("cp.async.commit_group;" ::: "memory"); }
  // all copies but those of the stages - 1 youngest tiles have arrived
  __device__ __forceinline__ void wait(int stages) const {
    if (stages == 3) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else asm volatile("cp.async.wait_group 1;" ::: "memory");
  }
};

// Forward: at most 80 registers a thread, so that 768 threads fit an SM; backward: 128 and 512.
constexpr int NORM_FWD_REGS = 80, NORM_FWD_THREADS = 768, NORM_BWD_REGS = 128, NORM_BWD_THREADS = 512;

// Forward.  JOIN false: prenorm of X.  Blocks walk tiles of RPB rows in strides, with the gains in registers.
template <class T, int NV, bool RING, bool JOIN>
__global__ void __maxnreg__(NV > 2 ? 128 : NORM_FWD_REGS)
norm_fwd_kernel(const NormArgs p, const RowShape sh) {
  constexpr int P = PIECE<T>, NT = JOIN ? 2 : 1;
  extern __shared__ uint4 ring_smem[];
  __shared__ float red[2][NORM_MAX_WARPS];
  RowSum row_sum{red, sh.tpr, 0};
  const RowRing<NT, NV> ring{ring_smem};
  const int TPR = sh.tpr, RPB = sh.rpb, S = sh.stages;
  const int row = threadIdx.x / TPR, tg = threadIdx.x - row * TPR, np = p.d / P;
  const float inv_d = 1.f / (float)p.d;
  const long long step = (long long)gridDim.x * RPB;
  auto fetch = [&](int stage, long long t) {
    if (t < p.T) {
      const size_t off = (size_t)t * np;
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const int g = tg + u * TPR;
        if (g >= np) continue;
        if (JOIN) ring.fetch(stage, NT - 1, u, (const uint4*)p.Y + off + g);
        ring.fetch(stage, 0, u, (const uint4*)p.X + off + g);
      }
    }
    ring.commit();
  };
  grid_sync();
  long long t = (long long)blockIdx.x * RPB + row;
  if (RING)
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
    if (RING) {
      fetch(stage == 0 ? S - 1 : stage - 1, t + (S - 1) * step);
      ring.wait(S);
    }
    auto piece = [&](int tensor, const void* base, int u) {
      const int g = tg + u * TPR;
      if (!live || g >= np) return make_uint4(0, 0, 0, 0);
      return RING ? *ring.slot(stage, tensor, u) : ((const uint4*)base)[off + g];
    };
    float x[NV][P];
#pragma unroll
    for (int u = 0; u < NV; ++u) unpack<T>(piece(0, p.X, u), x[u]);
    if (JOIN) {
      float y[NV][P], f = p.b * gate;
#pragma unroll
      for (int u = 0; u < NV; ++u) unpack<T>(piece(NT - 1, p.Y, u), y[u]);
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
    stage = stage + 1 < S ? stage + 1 : 0;
  }
}

// Backward.  Blocks walk tiles of RPB rows in strides, a thread always on the same columns, so the gains' gradients add up in
// registers; a block leaves one row of partial sums per gain, which norm_dw_kernel adds in order.
// JOIN false: prenorm (Xo_in is its input X, dXo the gradient that comes along the residual, may be NULL; no y).
template <class T, int NV, bool RING, bool JOIN>
__global__ void __maxnreg__(NORM_BWD_REGS)
norm_bwd_kernel(const NormArgs p, const RowShape sh) {
  constexpr int P = PIECE<T>, NT = JOIN ? 4 : 3;
  extern __shared__ uint4 ring_smem[];
  __shared__ float red[2][NORM_MAX_WARPS];
  RowSum row_sum{red, sh.tpr, 0};
  const RowRing<NT, NV> ring{ring_smem};
  const int TPR = sh.tpr, RPB = sh.rpb, S = sh.stages;
  const int row = threadIdx.x / TPR, tg = threadIdx.x - row * TPR, np = p.d / P;
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
  if (RING)
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
    if (RING) {
      fetch(stage == 0 ? S - 1 : stage - 1, t + (S - 1) * step);
      ring.wait(S);
    }
    auto piece = [&](int tensor, const void* base, int u) {
      const int g = tg + u * TPR;
      if (base == nullptr || !live || g >= np) return make_uint4(0, 0, 0, 0);
      return RING ? *ring.slot(stage, tensor, u) : ((const uint4*)base)[off + g];
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
    stage = stage + 1 < S ? stage + 1 : 0;
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
      for (int c = threadIdx.x; c < p.d; c += blockDim.x) {
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

// Rows on threads.  2 pieces a thread where that is whole warps (one piece for rows within a warp), 4 or 8 where 512 threads
// would not hold the row; about 256 threads a block.
static int norm_pieces(int d, int dtype) { return d * (int)elem_bytes(dtype) / 16; }
static int norm_nv(int pieces) { return pieces <= 32 ? 1 : pieces <= 1024 ? 2 : pieces <= 2048 ? 4 : 8; }
static RowShape norm_shape(int pieces) {
  const int nv = norm_nv(pieces);
  RowShape s = {4, 1, 0};
  if (nv == 1)
    while (s.tpr < pieces) s.tpr *= 2;
  else
    s.tpr = ceil_div(pieces, 32 * nv) * 32;
  s.rpb = s.tpr < 256 ? 256 / s.tpr : 1;
  return s;
}

template <template <class, int> class K, class T>
static etr_status norm_by_shape(const NormArgs& p, cudaStream_t st) {
  const int pieces = p.d / PIECE<T>;
  const RowShape s = norm_shape(pieces);
  switch (norm_nv(pieces)) {
    case 1: return K<T, 1>::run(p, s, st);
    case 2: return K<T, 2>::run(p, s, st);
    case 4: return K<T, 4>::run(p, s, st);
  }
  return K<T, sizeof(T) == 2 ? 4 : 8>::run(p, s, st);      // 8: fp32 rows only
}
template <template <class, int> class K>
static etr_status norm_by_type(int dtype, const NormArgs& p, cudaStream_t st) {
  return dtype == ETR_BF16 ? norm_by_shape<K, __nv_bfloat16>(p, st) : norm_by_shape<K, float>(p, st);
}

// A ring of three tiles, or two, within the CTA's part of 200 KiB; 0: rows so long that two tiles do not fit are read without
// a ring.
static int ring_stages(long long tile, int ctas) {
  const long long n = 200 * 1024 / ctas / tile;
  return n < 2 ? 0 : n < 3 ? 2 : 3;
}

template <class K>
static etr_status norm_launch(const char* name, K kernel, std::atomic<unsigned long long>& done, size_t smem, int ctas, const NormArgs& p,
                              const RowShape& s, cudaStream_t st) {
  if (!ensure_dyn_smem(kernel, 200 * 1024, done)) return ETR_ERR_CUDA;
  const long long tiles = ((long long)p.T + s.rpb - 1) / s.rpb, most = (long long)current_sm_count() * ctas;
  ETR_TIME_BEGIN(name);
  launch_kernel(kernel, (unsigned)(tiles < most ? tiles : most), s.tpr * s.rpb, smem, st, 1, p, s);
  ETR_LAUNCH_CHECK();
  return ETR_OK;
}

template <class T, int NV>
struct FwdRun {
  template <bool JOIN>
  static etr_status go(const char* name, const NormArgs& p, RowShape s, cudaStream_t st) {
    static std::atomic<unsigned long long> done{0}, done0{0};
    const int block = s.tpr * s.rpb, threads = NV > 2 ? 512 : NORM_FWD_THREADS, ctas = threads / block > 1 ? threads / block : 1;
    const long long tile = (JOIN ? 2ll : 1ll) * NV * block * 16;
    s.stages = ring_stages(tile, ctas);
    if (NV > 2 && s.stages == 0) return norm_launch(name, norm_fwd_kernel<T, NV, NV <= 2, JOIN>, done0, 0, ctas, p, s, st);
    return norm_launch(name, norm_fwd_kernel<T, NV, true, JOIN>, done, (size_t)(s.stages * tile), ctas, p, s, st);
  }
  static etr_status run(const NormArgs& p, const RowShape& s, cudaStream_t st) {
    return p.Y ? go<true>("join_kernel", p, s, st) : go<false>("prenorm_kernel", p, s, st);
  }
};

static int norm_bwd_ctas(const RowShape& s) { return NORM_BWD_THREADS / (s.tpr * s.rpb) > 1 ? NORM_BWD_THREADS / (s.tpr * s.rpb) : 1; }
// Blocks of the backward kernels, each of which leaves a row of partial sums per gain; at most NORM_BWD_MOST an SM.
constexpr int NORM_BWD_MOST = 3;                  // blocks of 160 threads
static int norm_bwd_blocks(int T, int d, int dtype) {
  const RowShape s = norm_shape(norm_pieces(d, dtype));
  const long long want = ((long long)T + s.rpb - 1) / s.rpb, most = (long long)current_sm_count() * norm_bwd_ctas(s);
  return (int)(want < most ? want : most);
}

template <class T, int NV>
struct BwdRun {
  template <bool JOIN>
  static etr_status go(const char* name, const NormArgs& p, RowShape s, cudaStream_t st) {
    static std::atomic<unsigned long long> done{0}, done0{0};
    const int block = s.tpr * s.rpb, ctas = norm_bwd_ctas(s);
    const long long tile = (JOIN ? 4ll : 3ll) * NV * block * 16, fold = s.rpb > 1 ? (long long)s.rpb * p.d * 4 : 0;
    s.stages = ring_stages(tile, ctas);
    if (NV > 2 && s.stages == 0) return norm_launch(name, norm_bwd_kernel<T, NV, NV <= 2, JOIN>, done0, (size_t)fold, ctas, p, s, st);
    const long long smem = s.stages * tile;
    return norm_launch(name, norm_bwd_kernel<T, NV, true, JOIN>, done, (size_t)(smem > fold ? smem : fold), ctas, p, s, st);
  }
  static etr_status run(const NormArgs& p, const RowShape& s, cudaStream_t st) {
    return p.Y ? go<true>("join_bwd_kernel", p, s, st) : go<false>("prenorm_bwd_kernel", p, s, st);
  }
};

static etr_status norm_dw(const etr_norm_config* c, const NormArgs& p, float* dw_next, float* dw_post, cudaStream_t st) {
  if (dw_next == nullptr && dw_post == nullptr) return ETR_OK;
  const bool both = dw_next && dw_post;
  const float* a = dw_next ? p.part_next : p.part_post;
  ETR_TIME_BEGIN("norm_dw_kernel");
  launch_kernel(norm_dw_kernel, dim3(ceil_div(c->d, 32), both ? 2 : 1), 256, 0, st, 1, a, (const float*)p.part_post, dw_next ? dw_next : dw_post,
                dw_post, norm_bwd_blocks(c->T, c->d, c->dtype), c->d);
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
  *bytes = align_up((size_t)2 * current_sm_count() * NORM_BWD_MOST * c->d * 4, 256);
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
  p.part_post = dw_post ? (float*)ws + (size_t)current_sm_count() * NORM_BWD_MOST * c->d : nullptr;
  if (c->T > 0) ETR_TRY(norm_by_type<BwdRun>(c->dtype, p, (cudaStream_t)stream));
  return norm_dw(c, p, dw_next, dw_post, (cudaStream_t)stream);
}

}  // extern "C"
