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

__device__ __forceinline__ void load8(const float* w, int col, float* out) {       // w == nullptr: ones
  if (w) {
    const Vec8<float> q = Vec8<float>::load(w + col);
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = q.v[e];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) out[e] = 1.f;
  }
}

template <int TPR> constexpr int NORM_BLOCK = TPR > 256 ? TPR : 256;

// Forward.  A row is held in registers by TPR threads, NV groups of 8 values each.  JOIN false: prenorm of X.
template <class T, int TPR, int NV, bool JOIN>
__global__ void __launch_bounds__(NORM_BLOCK<TPR>)
norm_fwd_kernel(const NormArgs p) {
  constexpr int BLOCK = NORM_BLOCK<TPR>, RPB = BLOCK / TPR;
  __shared__ float red[2][BLOCK / 32];
  RowSum<TPR, BLOCK> row_sum{red, 0};
  grid_sync();
  const int tg = threadIdx.x % TPR, ng = p.d / 8;
  const long long t = (long long)blockIdx.x * RPB + threadIdx.x / TPR;
  const bool live = t < p.T;
  const size_t off = (size_t)(live ? t : 0) * p.d;
  float x[NV][8];
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int g = tg + u * TPR;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[u][e] = 0.f;
    if (!live || g >= ng) continue;
    const Vec8<T> q = Vec8<T>::load((const T*)p.X + off + g * 8);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[u][e] = q.v[e];
  }
  if (JOIN) {
    float y[NV][8], s = 0.f;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int g = tg + u * TPR;
#pragma unroll
      for (int e = 0; e < 8; ++e) y[u][e] = 0.f;
      if (!live || g >= ng) continue;
      const Vec8<T> q = Vec8<T>::load((const T*)p.Y + off + g * 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) { y[u][e] = q.v[e]; s = fmaf(q.v[e], q.v[e], s); }
    }
    float f = p.b;
    if (p.post) {
      s = row_sum(s);
      const float r = rsqrtf(s / (float)p.d + p.eps);
      if (p.rstd_y_out && live && tg == 0) p.rstd_y_out[t] = r;
      f *= r;
    }
    if (p.gate && live) f *= p.gate[t];
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int g = tg + u * TPR;
      if (!live || g >= ng) continue;
      float w[8];
      load8(p.w_post, g * 8, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[u][e] = fmaf(f * y[u][e], w[e], p.a * x[u][e]);
      Vec8<T>::store((T*)p.Xo + off + g * 8, x[u]);
    }
    if (p.N == nullptr) return;
  }
  float s = 0.f;
#pragma unroll
  for (int u = 0; u < NV; ++u)
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(x[u][e], x[u][e], s);
  s = row_sum(s);
  const float r = rsqrtf(s / (float)p.d + p.eps);
  if (p.rstd_o_out && live && tg == 0) p.rstd_o_out[t] = r;
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int g = tg + u * TPR;
    if (!live || g >= ng) continue;
    float w[8];
    load8(p.w_next, g * 8, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] *= x[u][e] * r;
    Vec8<T>::store((T*)p.N + off + g * 8, w);
  }
}

// Backward.  Blocks walk rows in strides, a thread always on the same columns, so the weights' gradients add up in
// registers; a block leaves one row of partial sums per weight, which norm_dw_kernel adds in order.
// JOIN false: prenorm (Xo_in is its input X, dXo the gradient that comes along the residual, may be NULL; no y).
template <class T, int TPR, int NV, bool JOIN>
__global__ void __launch_bounds__(NORM_BLOCK<TPR>)
norm_bwd_kernel(const NormArgs p) {
  constexpr int BLOCK = NORM_BLOCK<TPR>, RPB = BLOCK / TPR;
  __shared__ float red[2][BLOCK / 32];
  extern __shared__ float fold[];                // [RPB][d], only where a block has several rows
  RowSum<TPR, BLOCK> row_sum{red, 0};
  grid_sync();
  const int tg = threadIdx.x % TPR, row = threadIdx.x / TPR, ng = p.d / 8;
  const float inv_d = 1.f / (float)p.d;
  float acc_n[NV][8], acc_p[NV][8];
#pragma unroll
  for (int u = 0; u < NV; ++u)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc_n[u][e] = acc_p[u][e] = 0.f;
  for (long long tb = (long long)blockIdx.x * RPB; tb < p.T; tb += (long long)gridDim.x * RPB) {
    const long long t = tb + row;
    const bool live = t < p.T;
    const size_t off = (size_t)(live ? t : 0) * p.d;
    float G[NV][8];
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int g = tg + u * TPR;
#pragma unroll
      for (int e = 0; e < 8; ++e) G[u][e] = 0.f;
      if (!live || g >= ng || p.dXo == nullptr) continue;
      const Vec8<T> q = Vec8<T>::load((const T*)p.dXo + off + g * 8);
#pragma unroll
      for (int e = 0; e < 8; ++e) G[u][e] = q.v[e];
    }
    if (p.dN) {
      const float r = live ? p.rstd_o[t] : 0.f;
      float h[NV][8], gn[NV][8], s = 0.f;
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const int g = tg + u * TPR;
#pragma unroll
        for (int e = 0; e < 8; ++e) h[u][e] = gn[u][e] = 0.f;
        if (!live || g >= ng) continue;
        const Vec8<T> qn = Vec8<T>::load((const T*)p.dN + off + g * 8), qx = Vec8<T>::load((const T*)p.Xo_in + off + g * 8);
        float w[8];
        load8(p.w_next, g * 8, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          h[u][e] = qx.v[e] * r;
          acc_n[u][e] = fmaf(qn.v[e], h[u][e], acc_n[u][e]);
          gn[u][e] = qn.v[e] * w[e];
          s = fmaf(gn[u][e], h[u][e], s);
        }
      }
      s = row_sum(s) * inv_d;
#pragma unroll
      for (int u = 0; u < NV; ++u)
#pragma unroll
        for (int e = 0; e < 8; ++e) G[u][e] = fmaf(r, fmaf(-h[u][e], s, gn[u][e]), G[u][e]);
    }
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int g = tg + u * TPR;
      if (!live || g >= ng) continue;
      float out[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) out[e] = JOIN ? p.a * G[u][e] : G[u][e];
      Vec8<T>::store((T*)p.dX + off + g * 8, out);
    }
    if (JOIN) {
      const float r = p.post && live ? p.rstd_y[t] : 1.f;
      const float gate = p.gate && live ? p.gate[t] : 1.f;
      float h[NV][8], s = 0.f;
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const int g = tg + u * TPR;
#pragma unroll
        for (int e = 0; e < 8; ++e) h[u][e] = 0.f;
        if (!live || g >= ng) continue;
        const Vec8<T> q = Vec8<T>::load((const T*)p.Y + off + g * 8);
        float w[8];
        load8(p.w_post, g * 8, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          h[u][e] = q.v[e] * r;
          const float bg = p.b * G[u][e];
          acc_p[u][e] = fmaf(gate * bg, h[u][e], acc_p[u][e]);
          G[u][e] = bg * w[e];                               // b w_post G
          s = fmaf(G[u][e], h[u][e], s);
        }
      }
      s = row_sum(s);
      if (p.dgate && live && tg == 0) p.dgate[t] = s;
      const float c = p.post ? s * inv_d : 0.f, f = gate * r;
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const int g = tg + u * TPR;
        if (!live || g >= ng) continue;
        float out[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) out[e] = f * fmaf(-h[u][e], c, G[u][e]);
        Vec8<T>::store((T*)p.dY + off + g * 8, out);
      }
    }
  }
  // one row of partial sums per block and weight
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    float* part = which ? p.part_post : p.part_next;
    if (part == nullptr) continue;
    if (RPB > 1) __syncthreads();
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int g = tg + u * TPR;
      if (g >= ng) continue;
      float* dst = RPB > 1 ? fold + (size_t)row * p.d + g * 8 : part + (size_t)blockIdx.x * p.d + g * 8;
      Vec8<float>::store(dst, which ? acc_p[u] : acc_n[u]);
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

// Threads per row: as few as hold it with 2 groups of 8 values each, at least a warp, at most 512 (then 4 groups).
static int norm_tpr(int d) {
  int tpr = 32;
  while (tpr < 512 && d / 8 > 2 * tpr) tpr *= 2;
  return tpr;
}

template <template <class, int, int> class K, class T>
static etr_status norm_by_shape(const NormArgs& p, cudaStream_t st) {
  const int tpr = norm_tpr(p.d), nv = ceil_div(p.d / 8, tpr);
  switch (tpr) {
    case 32: return nv == 1 ? K<T, 32, 1>::run(p, st) : K<T, 32, 2>::run(p, st);
    case 64: return K<T, 64, 2>::run(p, st);
    case 128: return K<T, 128, 2>::run(p, st);
    case 256: return K<T, 256, 2>::run(p, st);
    default: return nv <= 2 ? K<T, 512, 2>::run(p, st) : K<T, 512, 4>::run(p, st);
  }
}
template <template <class, int, int> class K>
static etr_status norm_by_type(int dtype, const NormArgs& p, cudaStream_t st) {
  return dtype == ETR_BF16 ? norm_by_shape<K, __nv_bfloat16>(p, st) : norm_by_shape<K, float>(p, st);
}

template <class T, int TPR, int NV>
struct FwdRun {
  static etr_status run(const NormArgs& p, cudaStream_t st) {
    constexpr int block = NORM_BLOCK<TPR>;
    const unsigned grid = (unsigned)(((long long)p.T + block / TPR - 1) / (block / TPR));
    if (p.Y) {
      ETR_TIME_BEGIN("join_kernel");
      launch_kernel(norm_fwd_kernel<T, TPR, NV, true>, grid, block, 0, st, 1, p);
    } else {
      ETR_TIME_BEGIN("prenorm_kernel");
      launch_kernel(norm_fwd_kernel<T, TPR, NV, false>, grid, block, 0, st, 1, p);
    }
    ETR_LAUNCH_CHECK();
    return ETR_OK;
  }
};

constexpr int NORM_BWD_BLOCKS_PER_SM = 2;
static int norm_bwd_blocks(int T, int d) {
  const int tpr = norm_tpr(d), rpb = tpr < 256 ? 256 / tpr : 1;
  const long long want = ((long long)T + rpb - 1) / rpb, cap = (long long)current_sm_count() * NORM_BWD_BLOCKS_PER_SM;
  return (int)(want < cap ? want : cap);
}

template <class T, int TPR, int NV>
struct BwdRun {
  static etr_status run(const NormArgs& p, cudaStream_t st) {
    constexpr int block = NORM_BLOCK<TPR>, rpb = block / TPR;
    const unsigned grid = (unsigned)norm_bwd_blocks(p.T, p.d);
    const size_t smem = rpb > 1 ? (size_t)rpb * p.d * 4 : 0;          // at most 2 * 8 groups of 8 values a thread: 16 KiB
    if (p.Y) {
      ETR_TIME_BEGIN("join_bwd_kernel");
      launch_kernel(norm_bwd_kernel<T, TPR, NV, true>, grid, block, smem, st, 1, p);
    } else {
      ETR_TIME_BEGIN("prenorm_bwd_kernel");
      launch_kernel(norm_bwd_kernel<T, TPR, NV, false>, grid, block, smem, st, 1, p);
    }
    ETR_LAUNCH_CHECK();
    return ETR_OK;
  }
};

static etr_status norm_dw(const etr_norm_config* c, const NormArgs& p, float* dw_next, float* dw_post, cudaStream_t st) {
  if (dw_next == nullptr && dw_post == nullptr) return ETR_OK;
  const bool both = dw_next && dw_post;
  const float* a = dw_next ? p.part_next : p.part_post;
  ETR_TIME_BEGIN("norm_dw_kernel");
  launch_kernel(norm_dw_kernel, dim3(ceil_div(c->d, 32), both ? 2 : 1), 256, 0, st, 1, a, (const float*)p.part_post, dw_next ? dw_next : dw_post,
                dw_post, norm_bwd_blocks(c->T, c->d), c->d);
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
  *bytes = align_up((size_t)2 * current_sm_count() * NORM_BWD_BLOCKS_PER_SM * c->d * 4, 256);
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
  p.part_post = dw_post ? (float*)ws + (size_t)current_sm_count() * NORM_BWD_BLOCKS_PER_SM * c->d : nullptr;
  if (c->T > 0) ETR_TRY(norm_by_type<BwdRun>(c->dtype, p, (cudaStream_t)stream));
  return norm_dw(c, p, dw_next, dw_post, (cudaStream_t)stream);
}

}  // extern "C"
