// Tokens sorted by the expert a caller chose for them, and back: the plan (which row every (token, choice) pair takes) and
// the four row passes.  Stable: the rows of an expert hold its pairs in ascending (token, choice) order.
#include <cooperative_groups.h>

#include <algorithm>

#include "common.cuh"

namespace cg = cooperative_groups;

namespace etr {

constexpr int SORT_WARPS = 16;                   // at most
constexpr int SORT_CLUSTER = 8;                   // CTAs of a cluster, where there are several
constexpr int SORT_ALONE = 16;                    // CTAs at most of one that works alone
constexpr int SORT_MAX_CLUSTERS = 18;            // 144 of the 148 SMs
constexpr int SORT_ONE_CLUSTER = 65536;          // pairs that one cluster takes without a counting launch before it
constexpr int SORT_RUN = 32;                     // pairs per warp that are worth another CTA

struct SortShape {
  int N, k, E, align, capacity, stride, n_rows;      // stride: rows between experts in the capacity form, else 0
  int run;                                           // consecutive pairs per warp, whole rounds of 32
};

// Long batches, first of two launches: pairs per cluster and expert, part[cluster][E].  The same split over clusters as in
// sort_plan_kernel.
__global__ void __launch_bounds__(SORT_WARPS * 32)
sort_count_kernel(const int32_t* ids, SortShape s, int32_t* __restrict__ part) {
  grid_sync();
  extern __shared__ int mine[];                  // [E]
  cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, threads = blockDim.x;
  const int per = s.run * (threads >> 5);
  const long long beg = (long long)blockIdx.x * per, end = min((long long)s.N, beg + per);
  for (int e = tid; e < s.E; e += threads) mine[e] = 0;
  __syncthreads();
#pragma unroll 4
  for (long long i = beg + tid; i < end; i += threads) {
    const int e = ids[i];
    if ((unsigned)e < (unsigned)s.E) atomicAdd(&mine[e], 1);
  }
  cluster.sync();
  for (int e = (int)cluster.block_rank() * threads + tid; e < s.E; e += SORT_CLUSTER * threads) {
    int sum = 0;
#pragma unroll
    for (int c = 0; c < SORT_CLUSTER; ++c) sum += cluster.map_shared_rank(mine, c)[e];
    part[(size_t)(blockIdx.x / SORT_CLUSTER) * s.E + e] = sum;
  }
  cluster.sync();
}

// The plan.  Every warp owns a run of consecutive pairs and counts its ids per expert (shared memory); the warps' counts become
// prefix sums within the CTA, across the cluster (every CTA writes its counts to all others' shared memory, so that one
// barrier later all reads are local: 32768 pairs 5.6 us, 6.4 with counts read from there), and through `part` across the
// clusters (nclusters > 1).  The row of a pair is then its expert's start, plus the pairs of earlier warps, plus those before
// it in its own warp (one match over the warp's 32 ids a round).  No atomics decide an order, so the plan is stable and the
// same every time.  Bound by the latency of that chain, so a run's first SORT_KEPT rounds of ids stay in registers, loops over
// warps and CTAs are unrolled (their loads in flight together), and a short batch is one small CTA (64 x 2 ids 2.7 us).
constexpr int SORT_KEPT = 4;
__global__ void __launch_bounds__(SORT_WARPS * 32)
sort_plan_kernel(const int32_t* ids, SortShape s, const int32_t* part, int nclusters, int32_t* __restrict__ counts,
                 int32_t* __restrict__ offsets, int32_t* __restrict__ totals, int32_t* __restrict__ row_token,
                 int32_t* __restrict__ pos) {
  grid_sync();
  extern __shared__ int sm[];
  cg::cluster_group cluster = cg::this_cluster();
  const int threads = blockDim.x, warps = threads >> 5, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int ncta = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), my_cluster = blockIdx.x / ncta;
  int* wc = sm;                                  // [warps][E] pairs of this warp, then of the warps before it
  int* cta = wc + warps * s.E;                   // [CTAs][E] pairs of each CTA of the cluster, written by that CTA
  int* start = cta + ncta * s.E;                 // [E] first row of the expert
  int* before = start + s.E;                     // [E] pairs in the CTAs before this one
  int* used = before + s.E;                      // [E] pairs that get a row
  __shared__ int s_rows[SORT_WARPS], s_found[SORT_WARPS], s_kept[SORT_WARPS];
  if (ncta > 1) cluster.barrier_arrive();        // this CTA runs: the others may write to its memory
  const long long beg = ((long long)blockIdx.x * warps + warp) * s.run;
  const int n = (int)max(0ll, min((long long)s.run, (long long)s.N - beg));
  int id[SORT_KEPT];
#pragma unroll
  for (int u = 0; u < SORT_KEPT; ++u) id[u] = 32 * u + lane < n ? ids[beg + 32 * u + lane] : -1;
  int* cnt = wc + warp * s.E;
  for (int e = lane; e < s.E; e += 32) cnt[e] = 0;
  __syncwarp();
#pragma unroll
  for (int u = 0; u < SORT_KEPT; ++u)
    if ((unsigned)id[u] < (unsigned)s.E) atomicAdd(&cnt[id[u]], 1);
#pragma unroll 4
  for (int i = 32 * SORT_KEPT + lane; i < n; i += 32) {
    const int e = ids[beg + i];
    if ((unsigned)e < (unsigned)s.E) atomicAdd(&cnt[e], 1);
  }
  __syncthreads();
  if (ncta > 1) cluster.barrier_wait();
  for (int e = tid; e < s.E; e += threads) {
    int c[SORT_WARPS], acc = 0;
#pragma unroll
    for (int w = 0; w < SORT_WARPS; ++w) c[w] = w < warps ? wc[w * s.E + e] : 0;
#pragma unroll
    for (int w = 0; w < SORT_WARPS; ++w) {
      if (w < warps) wc[w * s.E + e] = acc;
      acc += c[w];
    }
    if (ncta == 1) {
      cta[e] = acc;
    } else {
      for (int q = 0; q < ncta; ++q) cluster.map_shared_rank(cta, q)[rank * s.E + e] = acc;
    }
  }
  if (ncta > 1) cluster.sync(); else __syncthreads();          // nothing goes to another CTA's memory behind this
  // Experts [2 tid, 2 tid + 2): pairs found, kept, and rows taken; the starts by a scan over the CTA's threads.
  int rows[2] = {0, 0}, found = 0, keeps = 0;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int e = 2 * tid + u;
    if (e >= s.E) break;
    int all = 0, ahead = 0;
#pragma unroll 8
    for (int c = 0; c < ncta; ++c) {
      const int v = cta[c * s.E + e];
      all += v;
      ahead += c < rank ? v : 0;
    }
    if (nclusters > 1) {
      all = 0;
#pragma unroll
      for (int c = 0; c < SORT_MAX_CLUSTERS; ++c) {
        const int v = c < nclusters ? part[(size_t)c * s.E + e] : 0;
        all += v;
        ahead += c < my_cluster ? v : 0;
      }
    }
    const int keep = s.capacity ? min(all, s.capacity) : all;
    before[e] = ahead;
    used[e] = keep;
    found += all;
    keeps += keep;
    rows[u] = s.capacity ? s.stride : (keep + s.align - 1) / s.align * s.align;
    if (blockIdx.x == 0) counts[e] = keep;
  }
  int inc = rows[0] + rows[1];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += y;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    found += __shfl_xor_sync(0xffffffffu, found, o);
    keeps += __shfl_xor_sync(0xffffffffu, keeps, o);
  }
  if (lane == 31) { s_rows[warp] = inc; s_found[warp] = found; s_kept[warp] = keeps; }
  __syncthreads();
  int at = inc - rows[0] - rows[1];
#pragma unroll
  for (int w = 0; w < SORT_WARPS; ++w) at += w < warp ? s_rows[w] : 0;
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int e = 2 * tid + u;
    if (e < s.E) {
      start[e] = at;
      if (blockIdx.x == 0) offsets[e] = at;
    }
    at += rows[u];
  }
  __syncthreads();
  const int limit = s.capacity ? s.capacity : s.N;
  for (int i0 = 0; i0 < n; i0 += 32 * SORT_KEPT) {
    if (i0 > 0) {
#pragma unroll
      for (int u = 0; u < SORT_KEPT; ++u) {
        const int i = i0 + 32 * u + lane;
        id[u] = i < n ? ids[beg + i] : -1;
      }
    }
#pragma unroll
    for (int u = 0; u < SORT_KEPT; ++u) {
      const int i = i0 + 32 * u + lane, e = id[u];
      if (i0 + 32 * u >= n) break;
      const bool ok = (unsigned)e < (unsigned)s.E;
      const unsigned same = __match_any_sync(0xffffffffu, ok ? e : -1);
      int r = 0;
      if (ok) r = cnt[e] + __popc(same & ((1u << lane) - 1u));
      __syncwarp();
      if (ok && (same >> lane) == 1u) cnt[e] = r + 1;         // the last of its kind in this round
      __syncwarp();
      if (i < n) {
        if (ok) r += before[e];
        const int row = ok && r < limit ? start[e] + r : -1;
        pos[beg + i] = row;
        if (row >= 0) row_token[row] = (int)((unsigned)(beg + i) / (unsigned)s.k);
      }
    }
  }
  // Rows without a token, an expert's at a time by one warp, or by several where there are more warps than experts; without
  // gaps between experts only those behind the last.
  const int first = s.align > 1 ? 0 : s.E - 1, spans = s.E - first, all_warps = gridDim.x * warps, gw = blockIdx.x * warps + warp;
  const int parts = max(1, all_warps / spans), share = gw / spans;           // parts > 1: one span a warp
#pragma unroll 4
  for (int x = parts > 1 ? gw - share * spans : gw; x < spans && (parts == 1 || share < parts); x += all_warps) {
    const int e = first + x;
    const int lo = start[e] + used[e], hi = e + 1 < s.E ? start[e + 1] : s.n_rows;
    const int lo4 = min((lo + 3) & ~3, hi), hi4 = max(hi & ~3, lo4);
    if (parts == 1 || share == 0) {
      if (lo + lane < lo4) row_token[lo + lane] = -1;
      if (hi4 + lane < hi) row_token[hi4 + lane] = -1;
    }
    // in 64 bits: a lane's first row and its step past the last one lie up to 128 * 2304 rows behind hi4, which may be near 2^31
    for (long long r = lo4 + 4ll * (lane + 32 * (parts > 1 ? share : 0)); r < hi4; r += 128ll * parts)
      *reinterpret_cast<int4*>(row_token + r) = make_int4(-1, -1, -1, -1);
  }
  if (blockIdx.x == 0 && tid == 0) {
    int end = 0, all = 0, with = 0;
    for (int w = 0; w < warps; ++w) { end += s_rows[w]; all += s_found[w]; with += s_kept[w]; }
    offsets[s.E] = end;
    totals[0] = with; totals[1] = all - with; totals[2] = s.N - all; totals[3] = 0;
  }
}

// Pad rows (behind an expert's last row, up to the next multiple of `align`) are zeros.  The first blocks of a row pass, one
// an expert for every 16 rows of `align` up to 8, write them, so that they do not end up as its tail.
__host__ __device__ constexpr int pad_shares(int align) { return align >= 128 ? 8 : (align + 15) / 16; }
__device__ __forceinline__ void zero_pad_rows(uint4* rows, int nv, const int32_t* counts, const int32_t* offsets, int align) {
  const int shares = pad_shares(align), e = blockIdx.x / shares, share = blockIdx.x % shares;
  const int c = counts[e], pads = (c + align - 1) / align * align - c;
  uint4* dst = rows + ((size_t)offsets[e] + c) * nv;
  const size_t n = (size_t)pads * nv;
  for (size_t v = share * 256 + threadIdx.x; v < n; v += shares * 256) dst[v] = make_uint4(0, 0, 0, 0);
}

// Xs[pos[t][j]] = X[t].  Token-major, so that a token is read once however many experts it has: HBM-bound, 65536 x 4096 bf16, k = 2
// 245 us, which is the copy rate (row-major, a token once per expert, would move a third more).  X is a flat run of 16-byte
// pieces; a thread takes U of them, and asks for the rows of AHEAD pairs of each (four, or k where that is fewer) before
// it stores (rows asked for one by one: 250 us, and 64 x 1024 2.5 us against 1.6).
constexpr int SORT_PIECES = 4;                   // U of batches that fill the SMs; 1 for shorter ones
template <int U, int AHEAD>
__global__ void __launch_bounds__(256)
sort_rows_kernel(const uint4* X, const int32_t* pos, const int32_t* counts, const int32_t* offsets, uint4* __restrict__ Xs, long long n,
                 int nv, int k, int align, int pad_blocks) {
  grid_sync();
  if ((int)blockIdx.x < pad_blocks) return zero_pad_rows(Xs, nv, counts, offsets, align);
  const long long base = (long long)(blockIdx.x - pad_blocks) * (256 * U);
  const long long t0 = base / nv;
  const int r0 = (int)(base - t0 * nv);
  const int32_t* p0 = pos + t0 * k;
  uint4 q[U];
  int v[U], first[U];                            // piece of the row, first pair from t0's on; -1: behind the end
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = u * 256 + (int)threadIdx.x;
    const unsigned dt = (unsigned)(r0 + i) / (unsigned)nv;
    v[u] = r0 + i - (int)dt * nv;
    first[u] = base + i < n ? (int)dt * k : -1;
    if (first[u] >= 0) q[u] = X[base + i];
  }
  for (int j0 = 0; j0 < k; j0 += AHEAD) {
    int r[U][AHEAD];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) r[u][j] = first[u] >= 0 && j0 + j < k ? p0[first[u] + j0 + j] : -1;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int j = 0; j < AHEAD; ++j)
        if (r[u][j] >= 0) Xs[(size_t)r[u][j] * nv + v[u]] = q[u];
  }
}

// Y[t] = sum_j w[t][j] rows[pos[t][j]], pairs without a row left out (w == nullptr: plain sum).  Sums in fp32, j ascending.  HBM-bound:
// what counts is loads in flight.  Any k: a 16-byte piece of a token a thread, four rows' pieces asked for before they are
// added (10 blocks of 128 threads an SM: 6113 x 2048 bf16, k = 8 34.1 us; 256 threads at 8, 6 and 5 blocks 40.8, 36.5, 34.7).
constexpr int UNSORT_THREADS = 128, UNSORT_AHEAD = 4;
template <class T>
__global__ void __launch_bounds__(UNSORT_THREADS, 10)
unsort_kernel(const uint4* rows, const float* w, const int32_t* pos, uint4* __restrict__ Y, long long n, int nv, int k) {
  constexpr int P = PIECE<T>, AHEAD = UNSORT_AHEAD;
  grid_sync();
  const long long base = (long long)blockIdx.x * UNSORT_THREADS;
  const long long t0 = base / nv;
  const int i = (int)(base - t0 * nv) + (int)threadIdx.x;
  if (base + (int)threadIdx.x >= n) return;
  const unsigned dt = (unsigned)i / (unsigned)nv;
  const int v = i - (int)dt * nv;
  const int32_t* p = pos + (t0 + dt) * k;
  const float* f = w ? w + (t0 + dt) * k : nullptr;
  rows += v;
  float acc[P];
#pragma unroll
  for (int e = 0; e < P; ++e) acc[e] = 0.f;
  for (int j0 = 0; j0 < k; j0 += AHEAD) {
    int r[AHEAD];
    uint4 q[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) r[u] = j0 + u < k ? p[j0 + u] : -1;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) q[u] = r[u] >= 0 ? rows[(size_t)r[u] * nv] : make_uint4(0, 0, 0, 0);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const float g = r[u] >= 0 && f ? f[j0 + u] : 1.f;
      float x[P];
      unpack<T>(q[u], x);
#pragma unroll
      for (int e = 0; e < P; ++e) acc[e] = fmaf(g, x[e], acc[e]);
    }
  }
  Y[base + (int)threadIdx.x] = pack<T>(acc);
}

// k <= 4 and pieces enough for every SM: U pieces of all K rows a thread, known to the compiler (16384 x 4096 bf16, k = 2 59.6 us
// against 77 in the form above, 20000 x 2048, k = 3 49.7 and 59; 28577 x 1632, k = 1 29.7 and 42).
__host__ __device__ constexpr int unsort_few_pieces(int k) { return k <= 2 ? 4 : k == 3 ? 2 : 1; }
template <class T, int K>
__global__ void __launch_bounds__(UNSORT_THREADS)
unsort_few_kernel(const uint4* rows, const float* w, const int32_t* pos, uint4* __restrict__ Y, long long n, int nv) {
  constexpr int P = PIECE<T>, U = unsort_few_pieces(K);
  grid_sync();
  const long long base = (long long)blockIdx.x * (UNSORT_THREADS * U);
  const long long t0 = base / nv;
  const int r0 = (int)(base - t0 * nv);
  uint4 q[U][K];
  float f[U][K];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int i = u * UNSORT_THREADS + (int)threadIdx.x;
    const unsigned dt = (unsigned)(r0 + i) / (unsigned)nv;
    const int v = r0 + i - (int)dt * nv;
#pragma unroll
    for (int j = 0; j < K; ++j) {
      const int r = base + i < n ? pos[(t0 + dt) * K + j] : -1;
      q[u][j] = r >= 0 ? rows[(size_t)r * nv + v] : make_uint4(0, 0, 0, 0);
      f[u][j] = r >= 0 && w ? w[(t0 + dt) * K + j] : 1.f;
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long long i = base + u * UNSORT_THREADS + threadIdx.x;
    if (i >= n) break;
    float acc[P];
#pragma unroll
    for (int e = 0; e < P; ++e) acc[e] = 0.f;
#pragma unroll
    for (int j = 0; j < K; ++j) {
      float x[P];
      unpack<T>(q[u][j], x);
#pragma unroll
      for (int e = 0; e < P; ++e) acc[e] = fmaf(f[u][j], x[e], acc[e]);
    }
    Y[i] = pack<T>(acc);
  }
}

// dO[pos[t][j]] = w[t][j] dY[t], dw[t][j] = <dY[t], O[pos[t][j]]>; L lanes per pair (a warp, or the power of two that holds a
// short row).  The pairs of a token are neighbours, so its dY comes from HBM once.  HBM-bound: 65536 x 4096 bf16, k = 2 400 us, the copy
// rate.
template <class T>
__global__ void __launch_bounds__(256)
unsort_bwd_kernel(const uint4* dY, const uint4* O, const float* w, const int32_t* pos, const int32_t* counts, const int32_t* offsets,
                  uint4* __restrict__ dO, float* __restrict__ dw, int pairs, int k, int nv, int L, int align, int pad_blocks) {
  constexpr int P = PIECE<T>, AHEAD = 4;
  grid_sync();
  if ((int)blockIdx.x < pad_blocks) return zero_pad_rows(dO, nv, counts, offsets, align);
  const long long i = ((long long)(blockIdx.x - pad_blocks) * 256 + threadIdx.x) / L;
  const int lane = threadIdx.x & (L - 1);
  const int row = i < pairs ? pos[i] : -1;
  float dot = 0.f;
  if (row >= 0) {
    const float f = w[i];
    const uint4* gy = dY + (size_t)(i / k) * nv;
    const uint4* o = O + (size_t)row * nv;
    uint4* out = dO + (size_t)row * nv;
    for (int v0 = lane; v0 < nv; v0 += L * AHEAD) {
      uint4 a[AHEAD], b[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        const bool in = v0 + u * L < nv;
        a[u] = in ? gy[v0 + u * L] : make_uint4(0, 0, 0, 0);
        b[u] = in ? o[v0 + u * L] : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        if (v0 + u * L >= nv) continue;
        float x[P], y[P];
        unpack<T>(a[u], x);
        unpack<T>(b[u], y);
#pragma unroll
        for (int e = 0; e < P; ++e) { dot = fmaf(x[e], y[e], dot); x[e] *= f; }
        out[v0 + u * L] = pack<T>(x);
      }
    }
  }
  for (int s = L >> 1; s > 0; s >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, s);
  if (lane == 0 && i < pairs) dw[i] = dot;
}

// The same for rows of at most 32 SHORT_STEPS pieces.  Such a pair is over so soon that a warp spends its time waiting for the
// pair's row number, then for the row; here blocks walk pairs in strides, the next pair's pieces are copied ahead into the
// lane's own slots of shared memory (cp.async) and the row of the one after it asked for.  7738 x 752 bf16, k = 4: 24.3 us
// as above, 19.2 so; but 16384 x 2048, k = 2: 51.7 as above, 55.8 with such a ring.
constexpr int SHORT_STEPS = 4, SHORT_SMEM = 2 * 2 * SHORT_STEPS * 256 * 16, SHORT_CTAS = 3;
template <class T>
__global__ void __launch_bounds__(256, SHORT_CTAS)
unsort_bwd_short_kernel(const uint4* dY, const uint4* O, const float* w, const int32_t* pos, const int32_t* counts, const int32_t* offsets,
                        uint4* __restrict__ dO, float* __restrict__ dw, int pairs, int k, int nv, int L, int align, int pad_blocks) {
  constexpr int P = PIECE<T>, N = SHORT_STEPS;
  grid_sync();
  if ((int)blockIdx.x < pad_blocks) return zero_pad_rows(dO, nv, counts, offsets, align);
  extern __shared__ uint4 slots[];
  const uint32_t mine = smem_u32(slots) + threadIdx.x * 16;        // slot (stage, tensor, u): (stage * 2 N + tensor * N + u) * 4096 on
  const int lane = threadIdx.x & (L - 1), per = 256 / L;
  const long long stride = (long long)(gridDim.x - pad_blocks) * per;
  long long i = (long long)(blockIdx.x - pad_blocks) * per + threadIdx.x / L;
  int row = i < pairs ? pos[i] : -1, row2 = i + stride < pairs ? pos[i + stride] : -1;
  float f = row >= 0 ? w[i] : 0.f;
  auto fetch = [&](int stage, long long at, int r) {
    if (r >= 0) {
      const uint4* gy = dY + (size_t)((unsigned)at / (unsigned)k) * nv + lane;
      const uint4* o = O + (size_t)r * nv + lane;
#pragma unroll
      for (int u = 0; u < N; ++u) {
        if (lane + u * L >= nv) break;
        const uint32_t dst = mine + (stage * 2 * N + u) * 4096;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(gy + u * L) : "memory");
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst + N * 4096), "l"(o + u * L) : "memory");
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  fetch(0, i, row);
  int stage = 0;
  for (long long base = i - (threadIdx.x & 31) / L; base < pairs; base += stride, i += stride, stage ^= 1) {      // base: the warp's first pair
    fetch(stage ^ 1, i + stride, row2);
    const float f2 = row2 >= 0 ? w[i + stride] : 0.f;
    const int row3 = i + 2 * stride < pairs ? pos[i + 2 * stride] : -1;
    asm volatile("cp.async.wait_group 1;" ::: "memory");
    float dot = 0.f;
    if (row >= 0) {
      uint4* out = dO + (size_t)row * nv + lane;
#pragma unroll
      for (int u = 0; u < N; ++u) {
        if (lane + u * L >= nv) break;
        uint4 a, b;
        const uint32_t src = mine + (stage * 2 * N + u) * 4096;
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w) : "r"(src) : "memory");
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w) : "r"(src + N * 4096) : "memory");
        float x[P], y[P];
        unpack<T>(a, x);
        unpack<T>(b, y);
#pragma unroll
        for (int e = 0; e < P; ++e) { dot = fmaf(x[e], y[e], dot); x[e] *= f; }
        out[u * L] = pack<T>(x);
      }
    }
    for (int s = L >> 1; s > 0; s >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, s);
    if (lane == 0 && i < pairs) dw[i] = dot;
    row = row2;
    row2 = row3;
    f = f2;
  }
}

// ---- launches ----------------------------------------------------------------------------------
static int sort_stride(const etr_sort_config* c) { return c->capacity ? (c->capacity + 127) / 128 * 128 : 0; }

static long long sort_rows_bound(const etr_sort_config* c) {
  if (c->capacity) return (long long)c->E * ((c->capacity + 127ll) / 128 * 128);
  const long long n = (long long)c->T * c->k;
  return n + (n < c->E ? n : c->E) * (long long)(c->align - 1);
}

static etr_status sort_valid(const etr_sort_config* c) {
  if (c == nullptr) return ETR_ERR_ARG;
  if (c->T < 0 || c->k < 1 || c->E < 1 || c->d < 1 || c->align < 1 || c->capacity < 0) return ETR_ERR_ARG;
  if (c->dtype != ETR_F32 && c->dtype != ETR_BF16) return ETR_ERR_ARG;
  if (c->k > ETR_SORT_MAX_K || c->E > ETR_SORT_MAX_E || c->d % 8 != 0 || c->align > 1024) return ETR_ERR_SHAPE;
  if (c->capacity && c->align != 128) return ETR_ERR_SHAPE;
  if ((long long)c->T * c->k >= (1ll << 31) - 65536 || sort_rows_bound(c) >= (1ll << 31) - 65536) return ETR_ERR_SHAPE;
  return ETR_OK;
}

static etr_status sort_plan_ptrs(const etr_sort_config* c, const etr_sort_plan* p, std::initializer_list<const void*> more) {
  if (p == nullptr || p->counts == nullptr || p->offsets == nullptr || p->totals == nullptr || p->scratch == nullptr) return ETR_ERR_ARG;
  const bool rows = sort_rows_bound(c) > 0, some = c->T > 0;
  if ((rows && p->row_token == nullptr) || (some && p->pos == nullptr)) return ETR_ERR_ARG;
  for (const int32_t* q : {p->counts, p->offsets, p->totals, p->row_token, p->pos, p->scratch})
    if (!aligned16(q)) return ETR_ERR_ALIGN;
  if (!some) return ETR_OK;                  // nothing is read or written through them
  for (const void* q : more) {
    if (q == nullptr) return ETR_ERR_ARG;
    if (!aligned16(q)) return ETR_ERR_ALIGN;
  }
  return ETR_OK;
}

etr_status sort_check_plan(const etr_sort_config* c, const etr_sort_plan* p) {
  ETR_TRY(sort_valid(c));
  return sort_plan_ptrs(c, p, {});
}

constexpr size_t SORT_SMEM = (size_t)(SORT_WARPS + SORT_ALONE + 3) * ETR_SORT_MAX_E * 4;        // of sort_plan_kernel, at most

// Clusters of more than 8 CTAs are allowed per kernel and device.
template <class K>
static bool ensure_wide_cluster(K kernel, std::atomic<unsigned long long>& done) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  const unsigned long long bit = 1ull << (dev & 63);
  if (done.load(std::memory_order_acquire) & bit) return true;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return false;
  done.fetch_or(bit, std::memory_order_release);
  return true;
}

static int sort_pad_blocks(const etr_sort_config* c) { return c->align > 1 ? pad_shares(c->align) * c->E : 0; }

// One cluster of as many CTAs as have SORT_RUN pairs a warp, up to 16 of 16 warps (an opt-in size); longer batches take up to
// 18 clusters of 8, and a launch before that counts the clusters' pairs.  Measured, a plan by itself: 32768 pairs of 32
// experts 5.6 us in one cluster of 16 (7.6 of 8, 9.5 with the count, before those counts were written instead of read); 65536 of
// 128 8.9 in one; 131072 of 64 9.4 with the count (14 without), 524288 16.  widest: CTAs of the widest cluster that the device
// takes; where that is less than a long batch's clusters have, one cluster takes any batch.
struct PlanSplit { int warps, ncta, nclusters; };
static PlanSplit plan_split(int pairs, int E, int widest) {
  const int cta = SORT_WARPS * SORT_RUN;
  if (pairs <= cta) {
    const int warps = std::max(std::max((pairs + 31) / 32, (E + 63) / 64), 4);
    return {std::min(warps, SORT_WARPS), 1, 1};
  }
  if (pairs > SORT_ONE_CLUSTER && widest >= SORT_CLUSTER)
    return {SORT_WARPS, SORT_CLUSTER, std::min(pairs / (cta * SORT_CLUSTER) + 1, SORT_MAX_CLUSTERS)};
  int ncta = 1;
  while (ncta < widest && pairs > ncta * cta) ncta *= 2;
  return {SORT_WARPS, ncta, 1};
}

// The widest cluster of the plan's kernel that the current device takes with the most shared memory that it can ask for, asked
// once per device: 16 CTAs on a whole B200, but a process may have been given fewer SMs of each GPC.
static int plan_widest() {
  static std::atomic<int> cache[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return SORT_ALONE;
  int n = cache[dev & 63].load(std::memory_order_relaxed);
  if (n > 0) return n;
  for (n = SORT_ALONE; n > 1; n /= 2) {
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = n; attr.val.clusterDim.y = 1; attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = n;
    cfg.blockDim = SORT_WARPS * 32;
    cfg.dynamicSmemBytes = SORT_SMEM;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    int clusters = 0;
    if (cudaOccupancyMaxActiveClusters(&clusters, sort_plan_kernel, &cfg) == cudaSuccess && clusters > 0) break;
    cudaGetLastError();
  }
  cache[dev & 63].store(n, std::memory_order_relaxed);
  return n;
}

static etr_status plan_launch(const etr_sort_config* c, const int32_t* ids, const etr_sort_plan* p, cudaStream_t st) {
  static std::atomic<unsigned long long> done{0}, wide{0};
  if (!ensure_dyn_smem(sort_plan_kernel, SORT_SMEM, done)) return ETR_ERR_CUDA;
  if (!ensure_wide_cluster(sort_plan_kernel, wide)) return ETR_ERR_CUDA;
  SortShape s{c->T * c->k, c->k, c->E, c->align, c->capacity, sort_stride(c), (int)sort_rows_bound(c), 0};
  const auto [warps, ncta, nclusters] = plan_split(s.N, s.E, plan_widest());
  const int all = warps * ncta * nclusters;
  s.run = ((s.N + all - 1) / all + 31) & ~31;
  if (nclusters > 1) {
    ETR_TIME_BEGIN("sort_count_kernel");
    launch_kernel(sort_count_kernel, nclusters * SORT_CLUSTER, SORT_WARPS * 32, (size_t)c->E * 4, st, SORT_CLUSTER, ids, s, p->scratch);
    ETR_LAUNCH_CHECK();
  }
  const size_t smem = (size_t)(warps + ncta + 3) * c->E * 4;
  ETR_TIME_BEGIN("sort_plan_kernel");
  launch_kernel(sort_plan_kernel, nclusters * ncta, warps * 32, smem, st, ncta, ids, s, (const int32_t*)p->scratch, nclusters, p->counts,
                p->offsets, p->totals, p->row_token, p->pos);
  ETR_LAUNCH_CHECK();
  return ETR_OK;
}

template <class T>
static etr_status sort_pass(int which, const etr_sort_config* c, const etr_sort_plan* p, const void* a, const void* b, const float* w,
                            void* out, float* dw, cudaStream_t st) {
  const int pad = sort_pad_blocks(c), nv = c->d / PIECE<T>;
  int L = 32;                                    // lanes per pair of unsort_bwd
  while (L > 1 && nv <= L / 2) L /= 2;
  const long long n = (long long)c->T * nv, pairs = (long long)c->T * c->k;
  const bool few = c->k <= 4 && n > (long long)current_sm_count() * 2048 * 2;      // two rounds of every SM's threads
  const int one = few ? UNSORT_THREADS * unsort_few_pieces(c->k) : UNSORT_THREADS;
  const bool full = n > (long long)current_sm_count() * 256 * SORT_PIECES;
  const int per = full ? 256 * SORT_PIECES : 256;
  long long blocks = which == 0 ? (n + per - 1) / per : which == 1 ? (n + one - 1) / one : (pairs * L + 255) / 256;
  const long long walk = (long long)current_sm_count() * SHORT_CTAS;
  const bool brief = which == 2 && nv <= 32 * SHORT_STEPS && blocks > walk;       // a walk of one pair gains nothing
  if (brief) blocks = walk;
  if (blocks + pad >= (1ll << 31)) return ETR_ERR_SHAPE;
  switch (which) {
    case 0:
      ETR_TIME_BEGIN("sort_rows_kernel");
      launch_kernel(!full ? sort_rows_kernel<1, 4> : c->k == 1 ? sort_rows_kernel<SORT_PIECES, 1> : c->k == 2 ? sort_rows_kernel<SORT_PIECES, 2>
                                                                                                 : sort_rows_kernel<SORT_PIECES, 4>,
                    (unsigned)(blocks + pad), 256, 0, st, 1, (const uint4*)a, p->pos, p->counts, p->offsets, (uint4*)out, n, nv, c->k, c->align, pad);
      break;
    case 1:
      ETR_TIME_BEGIN("unsort_kernel");
      if (few)
        launch_kernel(c->k == 1 ? unsort_few_kernel<T, 1> : c->k == 2 ? unsort_few_kernel<T, 2> : c->k == 3 ? unsort_few_kernel<T, 3>
                                                                                                 : unsort_few_kernel<T, 4>,
                      (unsigned)blocks, UNSORT_THREADS, 0, st, 1, (const uint4*)a, w, p->pos, (uint4*)out, n, nv);
      else
        launch_kernel(unsort_kernel<T>, (unsigned)blocks, UNSORT_THREADS, 0, st, 1, (const uint4*)a, w, p->pos, (uint4*)out, n, nv, c->k);
      break;
    case 2: {
      static std::atomic<unsigned long long> done{0};
      if (brief && !ensure_dyn_smem(unsort_bwd_short_kernel<T>, SHORT_SMEM, done)) return ETR_ERR_CUDA;
      ETR_TIME_BEGIN("unsort_bwd_kernel");
      launch_kernel(brief ? unsort_bwd_short_kernel<T> : unsort_bwd_kernel<T>, (unsigned)(blocks + pad), 256, brief ? (size_t)SHORT_SMEM : 0, st, 1,
                    (const uint4*)a, (const uint4*)b, w, p->pos, p->counts, p->offsets, (uint4*)out, dw, (int)pairs, c->k, nv, L, c->align, pad);
      break;
    }
  }
  ETR_LAUNCH_CHECK();
  return ETR_OK;
}

static etr_status sort_pass_typed(int which, const etr_sort_config* c, const etr_sort_plan* p, const void* a, const void* b, const float* w,
                                  void* out, float* dw, cudaStream_t st) {
  if (c->T == 0) return ETR_OK;
  return c->dtype == ETR_BF16 ? sort_pass<__nv_bfloat16>(which, c, p, a, b, w, out, dw, st) : sort_pass<float>(which, c, p, a, b, w, out, dw, st);
}

}  // namespace etr

using namespace etr;

extern "C" {

etr_status etr_sort_validate(const etr_sort_config* c) { return sort_valid(c); }

int64_t etr_sort_n_rows(const etr_sort_config* c) { return sort_valid(c) == ETR_OK ? sort_rows_bound(c) : 0; }

etr_status etr_sort_plan_bind(const etr_sort_config* c, void* base, size_t bytes, etr_sort_plan* out, size_t* need) {
  ETR_TRY(sort_valid(c));
  if (need == nullptr && out == nullptr) return ETR_ERR_ARG;
  if (out && base == nullptr) return ETR_ERR_ARG;
  if (out && (reinterpret_cast<uintptr_t>(base) & 255u)) return ETR_ERR_ALIGN;
  size_t off = 0;
  auto take = [&](size_t n) { char* q = (char*)base + off; off = align_up(off + n * 4, 256); return (int32_t*)q; };
  etr_sort_plan p;
  p.counts = take(c->E);
  p.offsets = take(c->E + 1);
  p.totals = take(4);
  p.row_token = take((size_t)sort_rows_bound(c));
  p.pos = take((size_t)c->T * c->k);
  p.scratch = take((size_t)SORT_MAX_CLUSTERS * c->E);
  if (need) *need = off;
  if (out) {
    if (bytes < off) return ETR_ERR_WORKSPACE;
    *out = p;
  }
  return ETR_OK;
}

etr_status etr_sort(const etr_sort_config* c, const int32_t* topk_idx, const etr_sort_plan* plan, void* stream) {
  ETR_TRY(sort_valid(c));
  ETR_TRY(sort_plan_ptrs(c, plan, {topk_idx}));
  return plan_launch(c, topk_idx, plan, (cudaStream_t)stream);
}

etr_status etr_sort_rows(const etr_sort_config* c, const void* X, const etr_sort_plan* plan, void* Xs, void* stream) {
  ETR_TRY(sort_valid(c));
  ETR_TRY(sort_plan_ptrs(c, plan, {X, Xs}));
  return sort_pass_typed(0, c, plan, X, nullptr, nullptr, Xs, nullptr, (cudaStream_t)stream);
}

etr_status etr_sort_rows_bwd(const etr_sort_config* c, const void* dXs, const etr_sort_plan* plan, void* dX, void* stream) {
  ETR_TRY(sort_valid(c));
  ETR_TRY(sort_plan_ptrs(c, plan, {dXs, dX}));
  return sort_pass_typed(1, c, plan, dXs, nullptr, nullptr, dX, nullptr, (cudaStream_t)stream);
}

etr_status etr_unsort_rows(const etr_sort_config* c, const void* O, const float* weights, const etr_sort_plan* plan, void* Y, void* stream) {
  ETR_TRY(sort_valid(c));
  ETR_TRY(sort_plan_ptrs(c, plan, {O, weights, Y}));
  return sort_pass_typed(1, c, plan, O, nullptr, weights, Y, nullptr, (cudaStream_t)stream);
}

etr_status etr_unsort_rows_bwd(const etr_sort_config* c, const void* dY, const void* O, const float* weights, const etr_sort_plan* plan,
                               void* dO, float* dweights, void* stream) {
  ETR_TRY(sort_valid(c));
  ETR_TRY(sort_plan_ptrs(c, plan, {dY, O, weights, dO, dweights}));
  return sort_pass_typed(2, c, plan, dY, O, weights, dO, dweights, (cudaStream_t)stream);
}

}  // extern "C"
