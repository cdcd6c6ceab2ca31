// The norm before a block, and the join behind it: the block's output normed, gated, scaled and added to the scaled residual,
// with the next block's norm of the sum; forward and backward.  A row is d values; r(x) = 1 / sqrt(mean x^2 + eps).
//   prenorm  N = x r(x) w
//   join     v = y r(y) w_post (or y w_post),  Xo = a X + b gate v,  N = Xo r(Xo) w_next
// Backward, with xh = Xo r_o, yh = y r_y and <,> the sum over a row:
//   G = dXo + r_o (w_next dN - xh <w_next dN, xh> / d),   dX = a G,   dgate = b <G, w_post yh>
//   u = b gate w_post G,   dY = r_y (u - yh <u, yh> / d),   dw_post = sum_t b gate G yh,   dw_next = sum_t dN xh
// All sums in fp32; a row's norm is taken of the unrounded fp32 sum.
#include <cooperative_groups.h>

#include "common.cuh"

namespace cg = cooperative_groups;

namespace etr {

struct NormArgs {
  const void *X, *Y, *dXo, *dN, *Xo_in;          // X: input of prenorm, residual of join; Xo_in: the saved sum (backward)
  const float *w_post, *w_next, *gate, *rstd_y, *rstd_o;
  void *Xo, *N, *dX, *dY;
  float *rstd_y_out, *rstd_o_out, *dgate, *part_post, *part_next, *dw_post, *dw_next;
  int T, d, post;
  float eps, a, b;
};

// How rows lie on a block's threads: tpr threads hold a row (a power of two up to 32, or whole warps), NV pieces of 16 bytes each
// (piece u of a thread is piece tg + u tpr of the row), rpb rows side by side in a block.
// alone: the grid is one cluster, which adds its blocks' gradients of the gains by itself (backward of short batches).
struct RowShape { int tpr, rpb, alone; };

// Sum over a row's threads, in every one of them.  Two arrays take turns from sum to sum, so that one barrier a sum is
// enough: whoever writes an array again has passed the barrier of the sum between, and so has every reader.
constexpr int NORM_MAX_WARPS = 16;                // of a row, 512 threads
constexpr int NORM_WIDE_ROWS = 4;                 // rows of more than a warp in a block of about 256 threads
struct RowSum {
  float (*red)[NORM_WIDE_ROWS][NORM_MAX_WARPS];   // [2][rows][warps of a row], zeros behind a row's last warp
  int tpr, row, turn;
  __device__ __forceinline__ void init() {
    if (tpr <= 32) return;
    for (int i = threadIdx.x; i < 2 * NORM_WIDE_ROWS * NORM_MAX_WARPS; i += blockDim.x) (&red[0][0][0])[i] = 0.f;
    __syncthreads();
  }
  __device__ __forceinline__ float operator()(float v) {
    if (tpr <= 32) {
      for (int o = tpr >> 1; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
      return v;
    }
    v = warp_sum(v);
    const int wpr = tpr >> 5;
    float* mine = red[turn][row];
    if ((threadIdx.x & 31) == 0) mine[(threadIdx.x >> 5) - row * wpr] = v;
    __syncthreads();
    const float4* q = reinterpret_cast<const float4*>(mine);
    float4 s = q[0];
    v = (s.x + s.y) + (s.z + s.w);
    if (wpr > 4) {
      s = q[1];
      v += (s.x + s.y) + (s.z + s.w);
      if (wpr > 8) {
        const float4 a = q[2], c = q[3];
        v += ((a.x + a.y) + (a.z + a.w)) + ((c.x + c.y) + (c.z + c.w));
      }
    }
    turn ^= 1;
    return v;
  }
};

// Two fp32 values a register pair and instruction (fma.rn.f32x2 and its kin): these kernels are bound by the instructions
// they issue, not by the multipliers.
__device__ __forceinline__ unsigned long long bits2(float2 v) { return *reinterpret_cast<unsigned long long*>(&v); }
__device__ __forceinline__ float2 from2(unsigned long long v) { return *reinterpret_cast<float2*>(&v); }
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  unsigned long long r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)), "l"(bits2(c)));
  return from2(r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)));
  return from2(r);
}
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

template <class T>
__device__ __forceinline__ void unpack2(const uint4 q, float2* v) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
  if (sizeof(T) == 4) {
    v[0] = make_float2(__uint_as_float(w[0]), __uint_as_float(w[1]));
    v[1] = make_float2(__uint_as_float(w[2]), __uint_as_float(w[3]));
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[sizeof(T) == 4 ? 0 : i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
  }
}
template <class T>
__device__ __forceinline__ uint4 pack2(const float2* v) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (sizeof(T) == 4) {
      w[i] = __float_as_uint(i & 1 ? v[i / 2].y : v[i / 2].x);
    } else {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[sizeof(T) == 4 ? 0 : i].x, v[sizeof(T) == 4 ? 0 : i].y);
      w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
template <int H>                                  // H pairs from column col on; w == nullptr: ones
__device__ __forceinline__ void load_gain(const float* w, int col, float2* out) {
#pragma unroll
  for (int e = 0; e < H; e += 2) {
    const float4 q = w ? *reinterpret_cast<const float4*>(w + col + 2 * e) : make_float4(1.f, 1.f, 1.f, 1.f);
    out[e] = make_float2(q.x, q.y);
    out[e + 1] = make_float2(q.z, q.w);
  }
}

// The rows of up to NT tensors, one tile ahead of their use.  A thread copies (cp.async) exactly the pieces that it reads
// itself, so that a wait for its own copies is all the synchronisation the ring needs.  Pieces behind a row's end and rows
// behind the last arrive as zeros (a copy of no bytes).  A second tile ahead cost time (bf16: prenorm of 65536 x 4096 167 us
// with one, 188 with two; join backward of 16384 x 4096 137 and 145).  RING false: rows so long that two tiles do not
// fit shared memory come straight from global memory (join backward from d > 12288 in bf16 and d > 6144 in fp32 on, prenorm backward
// from d > 8192 and join from d > 12288 on, both in fp32).
template <int NT, int NV, bool RING>
struct RowRing {
  uint32_t smem;                                  // this thread's first slot
  uint32_t pitch;                                 // between pieces, 16 bytes a thread
  int stage;
  __device__ __forceinline__ uint32_t slot(int st, int tensor, int u) const { return smem + ((st * NT + tensor) * NV + u) * pitch; }
  __device__ __forceinline__ void fetch(int st, int tensor, int u, const uint4* src, bool there) const {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(slot(st, tensor, u)), "l"(src), "r"(there ? 16 : 0) : "memory");
  }
  __device__ __forceinline__ void commit() const { asm volatile("cp.async.commit_group;" ::: "memory"); }
  // all copies but those of the youngest tile have arrived
  __device__ __forceinline__ void wait() const { asm volatile("cp.async.wait_group 1;" ::: "memory"); }
  __device__ __forceinline__ uint4 piece(int tensor, int u, const void* base, size_t at, bool there) const {
    if (RING) {
      uint4 q;
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w) : "r"(slot(stage, tensor, u)) : "memory");
      return q;
    }
    return there ? ((const uint4*)base)[at] : make_uint4(0, 0, 0, 0);
  }
};

// Threads of an SM, which is what the launch bounds ask for (a block has at most 512): forward 768 with at most 80 registers each,
// and 1024 with 64 for a prenorm whose block is more than 384 threads, so that two fit (fp32 40920 x 3280: 72 % of the copy
// rate with one, 97 with two; smaller blocks lose: 20000 x 1088 bf16 75 and 67 %); prenorm's backward 576 with 112, which fits a
// third block of 192 threads (20000 x 1088: 49 % with two, 76 with three); the join's backward, and rows of more than 2
// pieces a thread, 512 with 128 (the join's spills at 112).  128 registers do not hold the gains and their gradients of every row of more
// than 2 pieces: the join's backward spills 304 to 312 bytes a thread in bf16 (d > 8192) and 428 in fp32 (d > 8192), prenorm's
// 24 in bf16.  Of the copy rate, at 2^27 values: join backward bf16 d = 8192 95 %, 10240 to 16384 37 to 54; fp32 6144 93, 8192 (no
// ring) 66, 12288 to 16384 41 to 46; prenorm backward bf16 8192 100, above 70 to 84; fp32 8192 99, above (no ring) 49 to 58;
// join fp32 12288 92, above (no ring) 54 to 63; all other forward forms 83 to 100.
constexpr int norm_bwd_threads(bool join, int nv) { return join || nv > 2 ? 512 : 576; }

// Forward.  JOIN false: prenorm of X.  Blocks walk tiles of rpb rows in strides, with the gains in registers.  HBM-bound: bf16, prenorm of
// 65536 x 4096 164 us (the copy rate), join of 65536 x 4096 347 us (94 %), of 6113 x 2048 17.8 us (86 %: seven tiles a block,
// ramp and tail); a few rows cost a launch (64 x 4096: join 2.5 us in a graph).
template <class T, int NV, bool RING, bool JOIN, int THREADS>
__global__ void __launch_bounds__(THREADS)
norm_fwd_kernel(const NormArgs p, const RowShape sh) {
  constexpr int P = PIECE<T>, H = P / 2, NT = JOIN ? 2 : 1, XX = 0, YY = NT - 1;
  grid_sync();
  extern __shared__ uint4 ring_smem[];
  __shared__ __align__(16) float red[2][NORM_WIDE_ROWS][NORM_MAX_WARPS];
  const int tpr = sh.tpr, row = threadIdx.x / tpr, tg = threadIdx.x - row * tpr, np = p.d / P;
  RowSum row_sum{red, tpr, row, 0};
  RowRing<NT, NV, RING> ring{smem_u32(ring_smem) + threadIdx.x * 16, blockDim.x * 16, 0};
  const float inv_d = 1.f / (float)p.d;
  const int step = gridDim.x * sh.rpb;
  const size_t stride = (size_t)step * np;
  bool in[NV];
#pragma unroll
  for (int u = 0; u < NV; ++u) in[u] = tg + u * tpr < np;
  auto fetch = [&](int st, long long tile, size_t at) {      // tile: its first row; at: this thread's first piece
    if (tile < p.T) {
      const bool live = tile + row < p.T;
      const size_t a = live ? at : 0;
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const size_t i = in[u] && live ? a + u * tpr : 0;
        if (JOIN) ring.fetch(st, YY, u, (const uint4*)p.Y + i, live && in[u]);
        ring.fetch(st, XX, u, (const uint4*)p.X + i, live && in[u]);
      }
    }
    ring.commit();
  };
  row_sum.init();
  long long tile = (long long)blockIdx.x * sh.rpb;
  size_t at = (size_t)(tile + row) * np + tg;
  if (RING) fetch(0, tile, at);
  float2 wp[JOIN ? NV : 1][H], wn[NV][H];
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int g = min(tg + u * tpr, np - 1);
    if (JOIN) load_gain<H>(in[u] ? p.w_post : nullptr, g * P, wp[u]);
    load_gain<H>(in[u] && p.N ? p.w_next : nullptr, g * P, wn[u]);
  }
  const bool gated = JOIN && p.gate != nullptr;
  float gate = gated && tile + row < p.T ? p.gate[tile + row] : 1.f;
  for (; tile < p.T; tile += step, at += stride, ring.stage ^= 1) {
    const long long t = tile + row;
    const bool live = t < p.T;
    if (RING) {
      fetch(ring.stage ^ 1, tile + step, at + stride);
      ring.wait();
    }
    float2 x[NV][H];
    if (JOIN) {
      float2 y[NV][H];
      float f = p.b * gate;
      if (gated && t + step < p.T) gate = p.gate[t + step];
#pragma unroll
      for (int u = 0; u < NV; ++u) unpack2<T>(ring.piece(YY, u, p.Y, at + u * tpr, live && in[u]), y[u]);
      if (p.post) {
        float2 s = both(0.f);
#pragma unroll
        for (int u = 0; u < NV; ++u)
#pragma unroll
          for (int e = 0; e < H; ++e) s = fma2(y[u][e], y[u][e], s);
        const float r = rsqrtf(row_sum(s.x + s.y) * inv_d + p.eps);
        if (p.rstd_y_out && live && tg == 0) p.rstd_y_out[t] = r;
        f *= r;
      }
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        unpack2<T>(ring.piece(XX, u, p.X, at + u * tpr, live && in[u]), x[u]);
#pragma unroll
        for (int e = 0; e < H; ++e) x[u][e] = fma2(mul2(y[u][e], both(f)), wp[u][e], mul2(x[u][e], both(p.a)));
        if (live && in[u]) ((uint4*)p.Xo)[at + u * tpr] = pack2<T>(x[u]);
      }
    } else {
#pragma unroll
      for (int u = 0; u < NV; ++u) unpack2<T>(ring.piece(XX, u, p.X, at + u * tpr, live && in[u]), x[u]);
    }
    if (p.N) {
      float2 s = both(0.f);
#pragma unroll
      for (int u = 0; u < NV; ++u)
#pragma unroll
        for (int e = 0; e < H; ++e) s = fma2(x[u][e], x[u][e], s);
      const float r = rsqrtf(row_sum(s.x + s.y) * inv_d + p.eps);
      if (p.rstd_o_out && live && tg == 0) p.rstd_o_out[t] = r;
#pragma unroll
      for (int u = 0; u < NV; ++u) {
#pragma unroll
        for (int e = 0; e < H; ++e) x[u][e] = mul2(mul2(x[u][e], both(r)), wn[u][e]);
        if (live && in[u]) ((uint4*)p.N)[at + u * tpr] = pack2<T>(x[u]);
      }
    }
  }
}

// Backward, HBM-bound: bf16, join of 65536 x 4096 486 to 531 us from box to box (92 to 100 %), prenorm of 16384 x 2048 45 us (90 %, 3 us of them
// norm_dw_kernel).  Blocks walk tiles of rpb rows in strides, a thread always on the same columns, so the gains' gradients add up in
// registers; a block leaves one row of partial sums per gain, which norm_dw_kernel adds in order.
// JOIN false: prenorm (Xo_in is its input X, dXo the gradient that comes along the residual, may be NULL; no y).
// The factors that are the same for a whole row (r_o, r_y, gate, a, b) are taken out of the sums over it:
//   s1 = <w_next dN, x>,  G = dXo + r_o w_next dN - (r_o^2 (r_o s1 / d)) x,   s2 = <w_post G, y>,  dgate = b r_y s2,
//   dY = (b gate r_y) w_post G - (b gate r_y (r_y (r_y s2 / d))) y
template <class T, int NV, bool RING, bool JOIN>
__global__ void __launch_bounds__(JOIN || NV > 2 ? 512 : 576)
norm_bwd_kernel(const NormArgs p, const RowShape sh) {
  constexpr int P = PIECE<T>, H = P / 2, NT = JOIN ? 4 : 3;
  enum { DN, XO, DXO, YY };
  grid_sync();
  extern __shared__ uint4 ring_smem[];
  __shared__ __align__(16) float red[2][NORM_WIDE_ROWS][NORM_MAX_WARPS];
  const int tpr = sh.tpr, row = threadIdx.x / tpr, tg = threadIdx.x - row * tpr, np = p.d / P;
  RowSum row_sum{red, tpr, row, 0};
  RowRing<NT, NV, RING> ring{smem_u32(ring_smem) + threadIdx.x * 16, blockDim.x * 16, 0};
  const float inv_d = 1.f / (float)p.d;
  const int step = gridDim.x * sh.rpb;
  const size_t stride = (size_t)step * np;
  bool in[NV];
#pragma unroll
  for (int u = 0; u < NV; ++u) in[u] = tg + u * tpr < np;
  auto fetch = [&](int st, long long tile, size_t at) {
    if (tile < p.T) {
      const bool live = tile + row < p.T;
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const bool there = live && in[u];
        const size_t i = there ? at + u * tpr : 0;
        if (p.dN) {
          ring.fetch(st, DN, u, (const uint4*)p.dN + i, there);
          ring.fetch(st, XO, u, (const uint4*)p.Xo_in + i, there);
        }
        if (p.dXo) ring.fetch(st, DXO, u, (const uint4*)p.dXo + i, there);
        if (JOIN) ring.fetch(st, YY, u, (const uint4*)p.Y + i, there);
      }
    }
    ring.commit();
  };
  row_sum.init();
  long long tile = (long long)blockIdx.x * sh.rpb;
  size_t at = (size_t)(tile + row) * np + tg;
  if (RING) fetch(0, tile, at);
  float2 wp[JOIN ? NV : 1][H], wn[NV][H], acc_p[JOIN ? NV : 1][H], acc_n[NV][H];
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int g = min(tg + u * tpr, np - 1);
    load_gain<H>(in[u] && p.dN ? p.w_next : nullptr, g * P, wn[u]);
    if (JOIN) load_gain<H>(in[u] ? p.w_post : nullptr, g * P, wp[u]);
#pragma unroll
    for (int e = 0; e < H; ++e) {
      acc_n[u][e] = both(0.f);
      if (JOIN) acc_p[u][e] = both(0.f);
    }
  }
  // a row's scalars are asked for one tile ahead
  float r_o = 0.f, r_y = 1.f, gate = 1.f;
  auto scalars = [&](long long t) {
    if (t >= p.T) return;
    if (p.dN) r_o = p.rstd_o[t];
    if (JOIN && p.post) r_y = p.rstd_y[t];
    if (JOIN && p.gate) gate = p.gate[t];
  };
  scalars(tile + row);
  for (; tile < p.T; tile += step, at += stride, ring.stage ^= 1) {
    const long long t = tile + row;
    const bool live = t < p.T;
    const float ro = r_o, ry = r_y, ga = gate;
    scalars(t + step);
    if (RING) {
      fetch(ring.stage ^ 1, tile + step, at + stride);
      ring.wait();
    }
    float2 G[NV][H];
    if (p.dN) {
      float2 s = both(0.f);
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        float2 x[H];
        unpack2<T>(ring.piece(DN, u, p.dN, at + u * tpr, live && in[u]), G[u]);
        unpack2<T>(ring.piece(XO, u, p.Xo_in, at + u * tpr, live && in[u]), x);
#pragma unroll
        for (int e = 0; e < H; ++e) {
          acc_n[u][e] = fma2(mul2(G[u][e], x[e]), both(ro), acc_n[u][e]);
          G[u][e] = mul2(G[u][e], wn[u][e]);
          s = fma2(G[u][e], x[e], s);
        }
      }
      const float c = -ro * (ro * (ro * row_sum(s.x + s.y) * inv_d));
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        float2 x[H], o[H];
        unpack2<T>(ring.piece(XO, u, p.Xo_in, at + u * tpr, live && in[u]), x);
        if (p.dXo) {
          unpack2<T>(ring.piece(DXO, u, p.dXo, at + u * tpr, live && in[u]), o);
#pragma unroll
          for (int e = 0; e < H; ++e) x[e] = fma2(x[e], both(c), o[e]);
        } else {
#pragma unroll
          for (int e = 0; e < H; ++e) x[e] = mul2(x[e], both(c));
        }
#pragma unroll
        for (int e = 0; e < H; ++e) G[u][e] = fma2(G[u][e], both(ro), x[e]);
      }
    } else {
#pragma unroll
      for (int u = 0; u < NV; ++u) unpack2<T>(ring.piece(DXO, u, p.dXo, at + u * tpr, live && in[u]), G[u]);
    }
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      float2 out[H];
#pragma unroll
      for (int e = 0; e < H; ++e) out[e] = JOIN ? mul2(G[u][e], both(p.a)) : G[u][e];
      if (live && in[u]) ((uint4*)p.dX)[at + u * tpr] = pack2<T>(out);
    }
    if (JOIN) {
      const float f = p.b * ga * ry;
      float2 s = both(0.f);
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        float2 y[H];
        unpack2<T>(ring.piece(YY, u, p.Y, at + u * tpr, live && in[u]), y);
#pragma unroll
        for (int e = 0; e < H; ++e) {
          acc_p[u][e] = fma2(mul2(G[u][e], y[e]), both(f), acc_p[u][e]);
          G[u][e] = mul2(G[u][e], wp[u][e]);
          s = fma2(G[u][e], y[e], s);
        }
      }
      const float s2 = ry * row_sum(s.x + s.y);
      if (p.dgate && live && tg == 0) p.dgate[t] = p.b * s2;
      const float c = p.post ? -f * (ry * (s2 * inv_d)) : 0.f;
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        float2 y[H];
        unpack2<T>(ring.piece(YY, u, p.Y, at + u * tpr, live && in[u]), y);
#pragma unroll
        for (int e = 0; e < H; ++e) y[e] = fma2(G[u][e], both(f), mul2(y[e], both(c)));
        if (live && in[u]) ((uint4*)p.dY)[at + u * tpr] = pack2<T>(y);
      }
    }
  }
  // One row of sums per block and gain.  Where a block has several rows, or the cluster is alone, they pass through the ring's
  // memory, [gain][row][d] (every copy into it has arrived: the last groups waited for are empty).
  float* fold = reinterpret_cast<float*>(ring_smem);
  const bool folds = sh.rpb > 1 || sh.alone;
  if (folds) __syncthreads();
#pragma unroll
  for (int which = 0; which < (JOIN ? 2 : 1); ++which) {
    float* part = which ? p.part_post : p.part_next;
    if (part == nullptr) continue;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      if (!in[u]) continue;
      const int g = (tg + u * tpr) * P;
      float* dst = folds ? fold + (size_t)(which * sh.rpb + row) * p.d + g : part + (size_t)blockIdx.x * p.d + g;
#pragma unroll
      for (int e = 0; e < H; e += 2) {
        const float2 *v = which ? acc_p[JOIN ? u : 0] : acc_n[u];
        *reinterpret_cast<float4*>(dst + 2 * e) = make_float4(v[e].x, v[e].y, v[e + 1].x, v[e + 1].y);
      }
    }
  }
  if (!folds) return;
  __syncthreads();
  const int quads = p.d / 4;
  if (sh.rpb > 1) {                              // a block's own rows, a thread four columns
    for (int i = threadIdx.x; i < (JOIN ? 2 : 1) * quads; i += blockDim.x) {
      const int which = i >= quads, c = i - which * quads;
      float* part = which ? p.part_post : p.part_next;
      if (part == nullptr) continue;
      float4* src = reinterpret_cast<float4*>(fold + (size_t)which * sh.rpb * p.d) + c;
      float4 s = src[0];
#pragma unroll 4
      for (int q = 1; q < sh.rpb; ++q) {
        const float4 v = src[(size_t)q * quads];
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
      }
      if (sh.alone) src[0] = s;
      else reinterpret_cast<float4*>(part + (size_t)blockIdx.x * p.d)[c] = s;
    }
  }
  if (!sh.alone) return;
  cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  const int blocks = (int)gridDim.x;
  for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < (JOIN ? 2 : 1) * quads; i += gridDim.x * blockDim.x) {
    const int which = i >= quads, c = i - which * quads;
    float* dw = which ? p.dw_post : p.dw_next;
    if (dw == nullptr) continue;
    float* src = fold + (size_t)which * sh.rpb * p.d + 4 * c;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int q = 0; q < blocks; ++q) {
      const float4 v = *reinterpret_cast<const float4*>(cluster.map_shared_rank(src, q));
      s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    reinterpret_cast<float4*>(dw)[c] = s;
  }
  cluster.sync();                                // no block leaves while another may still read its sums
}

// dw[c] = sum over the blocks' partial rows, in a fixed order; grid y: which weight.  A block has DW_THREADS / DW_COLS rows' places for
// DW_COLS columns (two sectors of 32 bytes a row), so that a thread's few loads are in flight together.  Beside 32 columns by
// 1024 threads: join backward of 441 x 7928 16.5 us and 18.0, prenorm backward of 203 x 2280 5.6 and 7.2.
constexpr int DW_COLS = 16, DW_THREADS = 512;
static_assert(DW_THREADS / 32 >= DW_COLS && DW_THREADS / 32 <= 32, "a warp a column in the last sum");
__global__ void __launch_bounds__(DW_THREADS)
norm_dw_kernel(const float* part0, const float* part1, float* __restrict__ dw0, float* __restrict__ dw1, int rows, int d) {
  grid_sync();
  __shared__ float red[DW_THREADS / 32][DW_COLS];
  const float* part = blockIdx.y ? part1 : part0;
  float* dw = blockIdx.y ? dw1 : dw0;
  const int col = threadIdx.x % DW_COLS, c = blockIdx.x * DW_COLS + col, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  float s = 0.f;
  if (c < d) {
#pragma unroll 4
    for (int r = threadIdx.x / DW_COLS; r < rows; r += DW_THREADS / DW_COLS) s += part[(size_t)r * d + c];
  }
#pragma unroll
  for (int o = 16; o >= DW_COLS; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if (lane < DW_COLS) red[warp][lane] = s;
  __syncthreads();
  if (warp < DW_COLS) {
    s = warp_sum(lane < DW_THREADS / 32 ? red[lane][warp] : 0.f);
    if (lane == 0 && blockIdx.x * DW_COLS + warp < d) dw[blockIdx.x * DW_COLS + warp] = s;
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

// Rows on threads.  2 pieces a thread, 4 or 8 where 512 threads would not hold the row; about 256 threads a block, or 128 where
// more threads fit an SM of `threads` then (three warps a row, join backward of 20000 x 1088: 71 and 75 % of the copy rate).
static int norm_pieces(int d, int dtype) { return d * (int)elem_bytes(dtype) / 16; }
static int norm_nv(int pieces) { return pieces <= 1024 ? 2 : pieces <= 2048 ? 4 : 8; }
static RowShape norm_shape(int pieces, int threads) {
  const int nv = norm_nv(pieces);
  RowShape s = {4, 1, 0};
  if (pieces <= 64)
    while (2 * s.tpr < pieces) s.tpr *= 2;
  else
    s.tpr = ceil_div(pieces, 32 * nv) * 32;
  const int wide = s.tpr < 256 ? 256 / s.tpr : 1, narrow = s.tpr < 128 ? 128 / s.tpr : 1;
  s.rpb = threads / (s.tpr * wide) * wide >= threads / (s.tpr * narrow) * narrow ? wide : narrow;
  return s;
}

template <template <class, int> class K, class T>
static etr_status norm_by_shape(const NormArgs& p, cudaStream_t st) {
  const int nv = norm_nv(p.d / PIECE<T>);
  return nv == 2 ? K<T, 2>::run(p, st) : nv == 4 ? K<T, 4>::run(p, st) : K<T, sizeof(T) == 2 ? 4 : 8>::run(p, st);      // 8: fp32 rows only
}
template <template <class, int> class K>
static etr_status norm_by_type(int dtype, const NormArgs& p, cudaStream_t st) {
  return dtype == ETR_BF16 ? norm_by_shape<K, __nv_bfloat16>(p, st) : norm_by_shape<K, float>(p, st);
}

static int norm_ctas(const RowShape& s, int threads) { return threads / (s.tpr * s.rpb) > 1 ? threads / (s.tpr * s.rpb) : 1; }
// Whether two tiles fit the CTA's part of 200 KiB.
static bool norm_ring(size_t tile, int ctas) { return 2 * tile * ctas <= 200 * 1024; }

// Rows of 2 pieces a thread always have a ring; those of more are one to a block of 288 to 512 threads.
constexpr bool always_ring(int slots, int nv) { return nv <= 2 || 2 * slots * 512 * 16 <= 200 * 1024; }
constexpr bool sometimes_ring(int slots, int nv) { return nv <= 2 || 2 * slots * 288 * 16 <= 200 * 1024; }

template <class K>
static etr_status norm_launch(const char* name, K kernel, std::atomic<unsigned long long>& done, size_t smem, int ctas, const NormArgs& p,
                              const RowShape& s, cudaStream_t st) {
  if (!ensure_dyn_smem(kernel, 200 * 1024, done)) return ETR_ERR_CUDA;
  const long long tiles = ((long long)p.T + s.rpb - 1) / s.rpb, most = (long long)current_sm_count() * ctas;
  ETR_TIME_BEGIN(name);
  launch_kernel(kernel, s.alone ? (unsigned)s.alone : (unsigned)(tiles < most ? tiles : most), s.tpr * s.rpb, smem, st, s.alone ? s.alone : 1, p, s);
  ETR_LAUNCH_CHECK();
  return ETR_OK;
}

template <class T, int NV>
struct FwdRun {
  template <bool JOIN>
  static etr_status go(const char* name, const NormArgs& p, cudaStream_t st) {
    if constexpr (NV == 2 && !JOIN)
      if (p.d / PIECE<T> > 768) return with<JOIN, 1024>(name, p, st);
    return with<JOIN, (NV > 2 ? 512 : 768)>(name, p, st);
  }
  template <bool JOIN, int THREADS>
  static etr_status with(const char* name, const NormArgs& p, cudaStream_t st) {
    const RowShape s = norm_shape(p.d / PIECE<T>, THREADS);
    const int ctas = norm_ctas(s, THREADS);
    constexpr int slots = (JOIN ? 2 : 1) * NV;
    const size_t tile = (size_t)slots * s.tpr * s.rpb * 16;
    if constexpr (!always_ring(slots, NV)) {
      static std::atomic<unsigned long long> done{0};
      if (!norm_ring(tile, ctas)) return norm_launch(name, norm_fwd_kernel<T, NV, false, JOIN, THREADS>, done, 0, ctas, p, s, st);
    }
    static std::atomic<unsigned long long> done{0};
    return norm_launch(name, norm_fwd_kernel<T, NV, true, JOIN, THREADS>, done, 2 * tile, ctas, p, s, st);
  }
  static etr_status run(const NormArgs& p, cudaStream_t st) { return p.Y ? go<true>("join_kernel", p, st) : go<false>("prenorm_kernel", p, st); }
};

// Blocks of the backward kernels, each of which leaves a row of partial sums per gain; at most NORM_BWD_MOST an SM.
constexpr int NORM_BWD_MOST = 5;                  // blocks of 96 threads
static int norm_bwd_blocks(int T, int d, int dtype, bool join) {
  const int pieces = norm_pieces(d, dtype), threads = norm_bwd_threads(join, norm_nv(pieces));
  const RowShape s = norm_shape(pieces, threads);
  const long long want = ((long long)T + s.rpb - 1) / s.rpb, most = (long long)current_sm_count() * norm_ctas(s, threads);
  return (int)(want < most ? want : most);
}

// Blocks of the cluster that does a short batch's backward pass by itself, gains' gradients included: a launch less.  0 for longer
// batches.  30 x 672 bf16, called one after another: prenorm backward 4.1 us in one launch, 5.8 to 6.7 in two (in a graph 3.7 and
// 4.0); clusters of 16 gained nothing more (64 x 1024: 4.5 us in a graph, 4.0 in two launches).
constexpr int NORM_ALONE = 8;
static int norm_alone(int T, int d, int dtype, bool join) {
  const int pieces = norm_pieces(d, dtype);
  const RowShape s = norm_shape(pieces, norm_bwd_threads(join, norm_nv(pieces)));
  const long long tiles = ((long long)T + s.rpb - 1) / s.rpb;
  int n = 1;
  while (n < tiles && n < NORM_ALONE) n *= 2;
  return tiles <= n ? n : 0;
}

template <class T, int NV>
struct BwdRun {
  template <bool JOIN>
  static etr_status go(const char* name, const NormArgs& p, cudaStream_t st) {
    constexpr int threads = norm_bwd_threads(JOIN, NV), slots = (JOIN ? 4 : 3) * NV;
    RowShape s = norm_shape(p.d / PIECE<T>, threads);
    if (p.part_next || p.part_post) s.alone = norm_alone(p.T, p.d, sizeof(T) == 2 ? ETR_BF16 : ETR_F32, JOIN);
    const int ctas = norm_ctas(s, threads);
    const size_t tile = (size_t)slots * s.tpr * s.rpb * 16, fold = s.rpb > 1 || s.alone ? (size_t)(JOIN ? 2 : 1) * s.rpb * p.d * 4 : 0;
    if constexpr (!always_ring(slots, NV)) {
      static std::atomic<unsigned long long> done{0};
      if (!norm_ring(tile, ctas)) return norm_launch(name, norm_bwd_kernel<T, NV, false, JOIN>, done, fold, ctas, p, s, st);
    }
    if constexpr (sometimes_ring(slots, NV)) {
      static std::atomic<unsigned long long> done{0};
      return norm_launch(name, norm_bwd_kernel<T, NV, true, JOIN>, done, 2 * tile > fold ? 2 * tile : fold, ctas, p, s, st);
    }
    return ETR_ERR_UNSUPPORTED;                  // not reached: a row of these sizes has a ring or has not
  }
  static etr_status run(const NormArgs& p, cudaStream_t st) { return p.Y ? go<true>("join_bwd_kernel", p, st) : go<false>("prenorm_bwd_kernel", p, st); }
};

static etr_status norm_dw(const etr_norm_config* c, bool join, const NormArgs& p, float* dw_next, float* dw_post, cudaStream_t st) {
  if (dw_next == nullptr && dw_post == nullptr) return ETR_OK;
  if (c->T > 0 && norm_alone(c->T, c->d, c->dtype, join)) return ETR_OK;             // the one cluster has written them
  const bool both = dw_next && dw_post;
  const float* a = dw_next ? p.part_next : p.part_post;
  ETR_TIME_BEGIN("norm_dw_kernel");
  launch_kernel(norm_dw_kernel, dim3(ceil_div(c->d, DW_COLS), both ? 2 : 1), DW_THREADS, 0, st, 1, a, (const float*)p.part_post,
                dw_next ? dw_next : dw_post, dw_post, norm_bwd_blocks(c->T, c->d, c->dtype, join), c->d);
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
  p.dw_next = dw;
  if (c->T > 0) ETR_TRY(norm_by_type<BwdRun>(c->dtype, p, (cudaStream_t)stream));
  return norm_dw(c, false, p, dw, nullptr, (cudaStream_t)stream);
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
  p.dw_next = dw_next;
  p.dw_post = dw_post;
  p.part_post = dw_post ? (float*)ws + (size_t)current_sm_count() * NORM_BWD_MOST * c->d : nullptr;
  if (c->T > 0) ETR_TRY(norm_by_type<BwdRun>(c->dtype, p, (cudaStream_t)stream));
  return norm_dw(c, true, p, dw_next, dw_post, (cudaStream_t)stream);
}

}  // extern "C"
