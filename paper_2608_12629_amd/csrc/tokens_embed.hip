// tokens_embed.hip -- rows of a token table and their gradient.
//
// Lookup: out_m = round(scale * W[t_m]), one pass, bound by HBM: each thread
// carries four rows' worth of one 16-byte column.
//
// Gradient: dW_v = round(scale * sum over the positions of v of G_m).
//   1. sort       positions by token, stable: by counting (rank_kernel) up to 8,192
//                 positions, else by the update's radix passes
//   2. clearing   of dW, beside the counting or after the passes
//   3. sums       slices of consecutive sorted positions add each token's rows in fp32 in
//                 that order; a run that a slice end cuts leaves its part in `carry`
//   4. cut runs   the slice where a run starts adds its parts in slice order
// No atomics on floating-point values: the same bits on every run.
#include <algorithm>
#include <type_traits>

#include "fkm_device.h"
#include "tokens_internal.h"

namespace fkm {

namespace {

// E elements of a row as fp32: 16 bytes where the row's start is aligned to them
// (VEC), else element by element with the row's end checked.
template <int DT> struct Tok {
  static constexpr int E = DT == DT_F32 ? 4 : 8;  // elements in 16 bytes
  using T = std::conditional_t<DT == DT_F32, float, uint16_t>;
  __device__ static float widen(T v) {
    if constexpr (DT == DT_F32) return v;
    else return Elem<DT>::widen(v);
  }
  __device__ static T narrow(float v) {
    if constexpr (DT == DT_F32) return v;
    else return Elem<DT>::narrow(v);
  }
};

template <int DT, bool VEC>
__device__ __forceinline__ uint4 load_raw(const typename Tok<DT>::T* row, int d, int D) {
  if constexpr (VEC) {
    return *reinterpret_cast<const uint4*>(row + d);
  } else {
    constexpr int E = Tok<DT>::E;
    alignas(16) typename Tok<DT>::T x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = d + e < D ? row[d + e] : typename Tok<DT>::T(0);
    return *reinterpret_cast<const uint4*>(x);
  }
}
template <int DT>
__device__ __forceinline__ void widen_e(const uint4& raw, float (&v)[Tok<DT>::E]) {
  constexpr int E = Tok<DT>::E;
  alignas(16) typename Tok<DT>::T x[E];
  *reinterpret_cast<uint4*>(x) = raw;
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = Tok<DT>::widen(x[e]);
}

// E elements (of type WT, which may hold them in 32 bytes) to a row.
template <int WT, int E, bool VEC>
__device__ __forceinline__ void store_e(typename Tok<WT>::T* row, int d, int D,
                                        const float (&v)[E]) {
  using T = typename Tok<WT>::T;
  alignas(16) T x[E];
#pragma unroll
  for (int e = 0; e < E; ++e) x[e] = Tok<WT>::narrow(v[e]);
  if constexpr (VEC) {
#pragma unroll
    for (int e = 0; e < E; e += 16 / (int)sizeof(T))
      *reinterpret_cast<uint4*>(row + d + e) = *reinterpret_cast<const uint4*>(x + e);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (d + e < D) row[d + e] = x[e];
  }
}

constexpr int EMB_U = 4;  // rows per thread
constexpr int64_t MAX_BLOCKS = 1 << 22;  // of 256 threads: a grid holds fewer than 2^32 threads

// tpr threads (a power of two) share a row.
template <int DT, bool VEC>
__global__ __launch_bounds__(256) void embed_kernel(const typename Tok<DT>::T* __restrict__ W,
                                                    const int32_t* __restrict__ idx, int64_t rows,
                                                    int64_t M, int V, int D, float scale, int tpr,
                                                    typename Tok<DT>::T* __restrict__ out) {
  constexpr int E = Tok<DT>::E;
  const int t = threadIdx.x, rpb = 256 / tpr;
  for (int64_t r0 = (int64_t)blockIdx.x * rpb * EMB_U + t / tpr; r0 < rows;
       r0 += (int64_t)gridDim.x * rpb * EMB_U) {
  int64_t src[EMB_U];
#pragma unroll
  for (int u = 0; u < EMB_U; ++u) {
    const int64_t r = r0 + u * rpb;
    const int id = r < rows ? idx[r] : -1;
    src[u] = (unsigned)id < (unsigned)V ? (r / M) * V + id : -1;
  }
  for (int d = (t % tpr) * E; d < D; d += tpr * E) {
    float v[EMB_U][E];
#pragma unroll
    for (int u = 0; u < EMB_U; ++u) {
      if (src[u] >= 0) {
        widen_e<DT>(load_raw<DT, VEC>(W + src[u] * D, d, D), v[u]);
#pragma unroll
        for (int e = 0; e < E; ++e) v[u][e] *= scale;
      } else {
#pragma unroll
        for (int e = 0; e < E; ++e) v[u][e] = 0.f;
      }
    }
#pragma unroll
    for (int u = 0; u < EMB_U; ++u)
      if (r0 + u * rpb < rows) store_e<DT, E, VEC>(out + (r0 + u * rpb) * D, d, D, v[u]);
  }
  }
}

template <int DT>
hipError_t launch_embed_dt(const void* W, const int32_t* idx, int64_t B, int64_t M, int64_t V,
                           int64_t D, float scale, void* out, hipStream_t s) {
  using T = typename Tok<DT>::T;
  constexpr int E = Tok<DT>::E;
  int tpr = 1;
  while (tpr < 256 && tpr * E < D) tpr *= 2;
  const int64_t rows = B * M, per = 256 / tpr * EMB_U;
  const dim3 grid((unsigned)std::min<int64_t>((rows + per - 1) / per, MAX_BLOCKS));
  if (D % E == 0)
    embed_kernel<DT, true><<<grid, 256, 0, s>>>((const T*)W, idx, rows, M, (int)V, (int)D, scale,
                                                tpr, (T*)out);
  else
    embed_kernel<DT, false><<<grid, 256, 0, s>>>((const T*)W, idx, rows, M, (int)V, (int)D, scale,
                                                 tpr, (T*)out);
  return hipGetLastError();
}

// ---- gradient ------------------------------------------------------------------
// 16 bytes of zeros a thread, at byte 16 i (bytes in all).
__device__ __forceinline__ void zero_at(char* p, int64_t bytes, int64_t i) {
  if (16 * i + 16 <= bytes) {
    *reinterpret_cast<uint4*>(p + 16 * i) = make_uint4(0, 0, 0, 0);
  } else {
    for (int64_t j = 16 * i; j < bytes; ++j) p[j] = 0;
  }
}
// (HBM takes 7 TB/s from many small workgroups; 4.4 from ones that clear 64 KiB each.)
__global__ __launch_bounds__(256) void zero_kernel(char* __restrict__ p, int64_t bytes, int64_t from) {
  zero_at(p, bytes, from + (int64_t)blockIdx.x * 256 + threadIdx.x);
}

// Positions sorted by token in one launch: a position's place is the number of positions
// with a smaller token, or with the same one further ahead.  A workgroup places 16
// positions; the tokens pass through LDS 4,096 at a time, and each lane counts those of
// its position over a 64th of them (a read brings four, a compare and an add-with-carry
// each).  9 us at 4,099 positions, 20 at 8,192; the radix passes 12 us each.  Workgroups past
// the first `nrank` clear dW.
constexpr int RANK_CHUNK = 4096, RANK_T = 1024, RANK_P = 16;
__global__ __launch_bounds__(RANK_T) void rank_kernel(const int32_t* __restrict__ idx, int M, int V,
                                                      int32_t* __restrict__ keys,
                                                      int32_t* __restrict__ perm,
                                                      int32_t* __restrict__ total, int nrank,
                                                      char* __restrict__ zero, int64_t bytes) {
  const int tid = threadIdx.x;
  if ((int)blockIdx.x >= nrank) {
    const int64_t per = gridDim.x - nrank;
    zero_at(zero, bytes, (blockIdx.y * per + blockIdx.x - nrank) * RANK_T + tid);
    return;
  }
  constexpr int NONE = 0x7fffffff, P = RANK_P, PARTS = RANK_T / P;
  __shared__ __attribute__((aligned(16))) int ids[RANK_CHUNK];
  __shared__ int place[P], valid;
  const int64_t b = blockIdx.y;
  idx += b * M;
  const int pl = tid % P, part = tid / P;  // the position and part of this lane
  const int p0 = blockIdx.x * P, p = p0 + pl;
  const int id = p < M ? idx[p] : -1;
  if (tid < P) place[tid] = 0;
  if (tid == 0) valid = 0;
  int cnt = 0;
  for (int c0 = 0; c0 < M; c0 += RANK_CHUNK) {
    __syncthreads();
    int nv = 0;
#pragma unroll
    for (int u = 0; u < RANK_CHUNK / RANK_T; ++u) {
      const int j = c0 + u * RANK_T + tid;
      const int v = j < M ? idx[j] : -1;
      const bool ok = (unsigned)v < (unsigned)V;
      ids[u * RANK_T + tid] = ok ? v : NONE;
      nv += __popcll(__ballot(ok));
    }
    if (blockIdx.x == 0 && (tid & 63) == 0) atomicAdd(&valid, nv);
    __syncthreads();
    // this lane's tokens: every PARTS-th four
    const int4* q = reinterpret_cast<const int4*>(ids);
    constexpr int N = RANK_CHUNK / 4 / PARTS;
    if (c0 + RANK_CHUNK <= p0 || c0 > p0) {  // all ahead of the positions, or none
      const int lim = c0 <= p0 ? id + 1 : id;
#pragma unroll 8
      for (int i = 0; i < N; ++i) {
        const int4 v = q[i * PARTS + part];
        cnt += v.x < lim;
        cnt += v.y < lim;
        cnt += v.z < lim;
        cnt += v.w < lim;
      }
    } else {
#pragma unroll 8
      for (int i = 0; i < N; ++i) {
        const int4 v = q[i * PARTS + part];
        const int ahead = p - (c0 + 4 * (i * PARTS + part));  // tokens of this four ahead of p
        cnt += v.x < id + (ahead > 0);
        cnt += v.y < id + (ahead > 1);
        cnt += v.z < id + (ahead > 2);
        cnt += v.w < id + (ahead > 3);
      }
    }
  }
  atomicAdd(&place[pl], cnt);
  __syncthreads();
  if (tid < P && (unsigned)id < (unsigned)V) {
    keys[b * M + place[tid]] = id;
    perm[b * M + place[tid]] = p;
  }
  if (blockIdx.x == 0 && tid == 0) total[b] = valid;
}

// The row of token v gets `acc` (times scale; added to what it holds).
template <int WT, int E, bool VEC>
__device__ __forceinline__ void put_row(typename Tok<WT>::T* row, int d, int D,
                                        const float (&acc)[E], float scale, bool accumulate) {
  float v[E];
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = acc[e] * scale;
  if (accumulate) {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (VEC || d + e < D) v[e] += Tok<WT>::widen(row[d + e]);
  }
  store_e<WT, E, VEC>(row, d, D, v);
}

// lpr lanes (one 16-byte column each) take a slice of `slice` sorted positions: all its
// rows are on their way, eight at a time, whatever tokens they belong to, and are added
// in order; where the token changes, the sum goes to its row of dW, or to `carry` (the
// slice's first or last) if the token's run goes on beyond the slice.
// Slices of 16 positions, or up to 128 while that leaves 4,096 waves: fewer cut runs.
int sum_lanes(int64_t chunks) {
  int lpr = 1;
  while (lpr < 64 && lpr < chunks) lpr *= 2;
  return lpr;
}
constexpr int64_t SUM_MIN = 16, SUM_MAX = 128;
int64_t sum_slice(int64_t B, int64_t M, int64_t chunks) {
  const int64_t lanes = sum_lanes(chunks) * ((chunks + 63) / 64);  // of a slice, all columns
  int64_t slice = SUM_MIN;
  while (slice < SUM_MAX && B * M / (2 * slice) * lanes >= 4096 * 64) slice *= 2;
  return slice;
}
template <int DT, int WT, bool VEC>
__global__ __launch_bounds__(256) void embed_sums_kernel(
    const typename Tok<DT>::T* __restrict__ G, const int32_t* __restrict__ keys,
    const int32_t* __restrict__ perm, const int32_t* __restrict__ total, int64_t M, int V, int D,
    int lpr, int slice, int nslices, float scale, int ncols, int accumulate,
    typename Tok<WT>::T* __restrict__ dW, float* __restrict__ carry) {
  constexpr int E = Tok<DT>::E, U = 8;
  const int64_t b = blockIdx.y, n = total[b];
  const int64_t w = ((int64_t)(blockIdx.x / ncols) * 256 + threadIdx.x) / lpr;
  const int64_t j0 = w * slice;
  // column blocks side by side: one of them at a time, over all rows, would meet only the
  // memory channels of that part of a row
  const int d = (blockIdx.x % ncols * lpr + threadIdx.x % lpr) * E;
  if (j0 >= n || d >= D) return;
  const int cnt = (int)min<int64_t>(n - j0, slice);
  keys += b * M + j0;
  perm += b * M + j0;
  G += b * M * D;
  dW += b * V * D;
  float* c = carry + (b * nslices + w) * 2 * D;
  const int before = j0 > 0 ? keys[-1] : -1, after = j0 + cnt < n ? keys[cnt] : -1;
  int key = keys[0];
  bool head = before == key;  // the run began in an earlier slice
  float acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = 0.f;
  auto flush = [&](bool tail) {
    if (head || tail) {
      float* o = c + (head ? 0 : D);
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (VEC || d + e < D) o[d + e] = acc[e];
    } else {
      put_row<WT, E, VEC>(dW + (int64_t)key * D, d, D, acc, scale, accumulate);
    }
  };
  for (int i0 = 0; i0 < cnt; i0 += U) {
    int k[U];
    uint4 raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) k[u] = keys[min(i0 + u, cnt - 1)];
#pragma unroll
    for (int u = 0; u < U; ++u)  // past the last one it again: no branch around a load
      raw[u] = load_raw<DT, VEC>(G + (int64_t)perm[min(i0 + u, cnt - 1)] * D, d, D);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u >= cnt) break;
      if (k[u] != key) {
        flush(false);
        key = k[u];
        head = false;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = 0.f;
      }
      float v[E];
      widen_e<DT>(raw[u], v);
#pragma unroll
      for (int e = 0; e < E; ++e) acc[e] += v[e];
    }
  }
  flush(after == key);
}

// The slice in which a cut run starts adds the run's parts in slice order, one wave per
// slice and 64 column chunks.  Runs over more than CUT_LONG slices (a token that a tenth
// of all positions hold) are then shared by the workgroup's 16 waves.
constexpr int CUT_T = 1024, CUT_LONG = 64;
template <int WT, int E, bool VEC>
__global__ __launch_bounds__(CUT_T) void embed_cut_kernel(
    const int32_t* __restrict__ keys, const int32_t* __restrict__ total, int64_t M, int V, int D,
    int slice, int nslices, float scale, int accumulate, const float* __restrict__ carry,
    typename Tok<WT>::T* __restrict__ dW) {
  constexpr int W = CUT_T / 64;
  __shared__ float part[W][64 * E];
  __shared__ int long_more[W];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t w0 = (int64_t)blockIdx.x * W, b = blockIdx.z;
  const int64_t n = total[b];
  if ((w0 + 1) * slice >= n) return;  // nothing after the first slice
  keys += b * M;
  const int d = (blockIdx.y * 64 + lane) * E;
  carry += b * nslices * 2 * D + d;
  // adds parts i0 + 1 .. i1 (the slices after w), all on their way eight at a time
  auto add = [&](float (&acc)[E], int64_t w, int i0, int i1) {
    constexpr int U = 8;
    const float* c = carry + w * 2 * D;
    for (; i0 < i1; i0 += U) {
      float v[U][E];
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int e = 0; e < E; ++e)
          v[u][e] = VEC || d + e < D ? c[(int64_t)min(i0 + u + 1, i1) * 2 * D + e] : 0.f;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i0 + u >= i1) break;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += v[u][e];
      }
    }
  };
  auto first = [&](float (&acc)[E], int64_t w) {
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = VEC || d + e < D ? carry[w * 2 * D + D + e] : 0.f;
  };
  {
    const int64_t w = w0 + wave, j0 = w * slice, j1 = j0 + slice;
    int more = 0;  // the slices that this slice's last run goes on into
    if (j1 < n && keys[j1] == keys[j1 - 1] && (j0 == 0 || keys[j0 - 1] != keys[j1 - 1])) {
      const int key = keys[j1 - 1];
      for (;;) {
        const int64_t j = j1 + (int64_t)(more + lane) * slice;
        const uint64_t on = ~__ballot(j < n && keys[j] == key);
        if (on) {
          more += (int)__builtin_ctzll(on);
          break;
        }
        more += 64;
      }
      if (more <= CUT_LONG && d < D) {
        float acc[E];
        first(acc, w);
        add(acc, w, 0, more);
        put_row<WT, E, VEC>(dW + (b * V + key) * D, d, D, acc, scale, accumulate);
      }
    }
    if (lane == 0) long_more[wave] = more > CUT_LONG ? more : 0;
  }
  __syncthreads();
  for (int i = 0; i < W; ++i) {
    const int more = long_more[i];
    if (!more) continue;
    float acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    if (d < D) {
      if (wave == 0) first(acc, w0 + i);
      add(acc, w0 + i, more * wave / W, more * (wave + 1) / W);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) part[wave][e * 64 + lane] = acc[e];
    __syncthreads();
    if (wave == 0 && d < D) {
      for (int q = 1; q < W; ++q)
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += part[q][e * 64 + lane];
      const int key = keys[(w0 + i + 1) * slice - 1];
      put_row<WT, E, VEC>(dW + (b * V + key) * D, d, D, acc, scale, accumulate);
    }
    __syncthreads();
  }
}

template <int DT, int WT, bool VEC>
hipError_t launch_sums_dt(const void* G, int64_t B, int64_t M, int64_t V, int64_t D, float scale,
                          bool accumulate, void* dW, const EmbedGradWs& w, hipStream_t s) {
  constexpr int E = Tok<DT>::E;
  const int64_t chunks = (D + E - 1) / E, slice = sum_slice(B, M, chunks);
  const int64_t nslices = (M + slice - 1) / slice;
  const int lpr = sum_lanes(chunks);
  using T = typename Tok<WT>::T;
  const int64_t ncols = (chunks + lpr - 1) / lpr;
  embed_sums_kernel<DT, WT, VEC>
      <<<dim3((unsigned)((nslices * lpr + 255) / 256 * ncols), (unsigned)B), 256, 0, s>>>(
          (const typename Tok<DT>::T*)G, w.sort.keys[0], w.sort.vals[0], w.sort.total, M, (int)V,
          (int)D, lpr, (int)slice, (int)nslices, scale, (int)ncols, accumulate, (T*)dW, w.carry);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || nslices == 1) return e;
  embed_cut_kernel<WT, E, VEC>
      <<<dim3((unsigned)((nslices + CUT_T / 64 - 1) / (CUT_T / 64)), (unsigned)((chunks + 63) / 64),
              (unsigned)B), CUT_T, 0, s>>>(
          w.sort.keys[0], w.sort.total, M, (int)V, (int)D, (int)slice, (int)nslices, scale,
          accumulate, w.carry,
          (T*)dW);
  return hipGetLastError();
}

template <int DT, int WT>
hipError_t launch_sums_wt(const void* G, int64_t B, int64_t M, int64_t V, int64_t D, float scale,
                          bool accumulate, void* dW, const EmbedGradWs& w, hipStream_t s) {
  return D % Tok<DT>::E == 0
             ? launch_sums_dt<DT, WT, true>(G, B, M, V, D, scale, accumulate, dW, w, s)
             : launch_sums_dt<DT, WT, false>(G, B, M, V, D, scale, accumulate, dW, w, s);
}

// ---- rows of no whole number of 16-byte chunks ----------------------------------------
struct PadJob {
  const uint16_t* in;
  uint4* out;
  int64_t chunks, total;  // 16-byte chunks of the copy, elements of the rows
};
constexpr int PAD_CHUNKS = 2048;  // of a workgroup

// A thread makes 16-byte chunks of the copy of 32-bit words, which start wherever a row
// does; the workgroups past the first nx are w's.  Bound by HBM: 43,047 rows of 1,331
// elements 43 us (5.3 TB/s read and written; with 64 rows to a workgroup 185).
__global__ __launch_bounds__(256) void pad_kernel(PadJob x, PadJob w, int D, int ch, int64_t nx) {
  const bool is_x = (int64_t)blockIdx.x < nx;
  const PadJob j = is_x ? x : w;
  const int64_t base = ((int64_t)blockIdx.x - (is_x ? 0 : nx)) * PAD_CHUNKS, row0 = base / ch;
  const uint32_t rem0 = (uint32_t)(base - row0 * ch);
  const uint32_t* words = reinterpret_cast<const uint32_t*>(j.in);
#pragma unroll 4
  for (int u = 0; u < PAD_CHUNKS / 256; ++u) {
    const uint32_t at = u * 256 + threadIdx.x, rem = rem0 + at, r = rem / (uint32_t)ch;
    if (base + at >= j.chunks) return;
    const int c = (int)(rem - r * ch) * 8, n = min(8, D - c);
    const int64_t e = (row0 + r) * D + c;
    uint32_t v[4];
    if (e + 9 <= j.total) {
      uint32_t x[5];
#pragma unroll
      for (int i = 0; i < 5; ++i) x[i] = i < 4 || (e & 1) ? words[(e >> 1) + i] : 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = e & 1 ? x[i] >> 16 | x[i + 1] << 16 : x[i];
        if (2 * i + 1 >= n) v[i] = 2 * i < n ? v[i] & 0xffffu : 0;  // the next row's
      }
    } else {  // the last chunks
#pragma unroll
      for (int i = 0; i < 4; ++i)
        v[i] = (2 * i < n ? j.in[e + 2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)j.in[e + 2 * i + 1] << 16 : 0u);
    }
    j.out[base + at] = make_uint4(v[0], v[1], v[2], v[3]);
  }
}

}  // namespace

hipError_t launch_pad_both(const void* X, int64_t xrows, void* xpad, const void* W, int64_t wrows,
                           void* wpad, int64_t D, hipStream_t s) {
  const int64_t ch = (D + 7) / 8;
  const PadJob x{(const uint16_t*)X, (uint4*)xpad, xrows * ch, xrows * D};
  const PadJob w{(const uint16_t*)W, (uint4*)wpad, wrows * ch, wrows * D};
  const int64_t nx = (x.chunks + PAD_CHUNKS - 1) / PAD_CHUNKS, nw = (w.chunks + PAD_CHUNKS - 1) / PAD_CHUNKS;
  pad_kernel<<<dim3((unsigned)(nx + nw)), 256, 0, s>>>(x, w, (int)D, (int)ch, nx);
  return hipGetLastError();
}

hipError_t launch_embed(const void* W, int dt, const int32_t* idx, int64_t B, int64_t M, int64_t V,
                        int64_t D, float scale, void* out, hipStream_t s) {
  if (dt == DT_BF16) return launch_embed_dt<DT_BF16>(W, idx, B, M, V, D, scale, out, s);
  if (dt == DT_F16) return launch_embed_dt<DT_F16>(W, idx, B, M, V, D, scale, out, s);
  return launch_embed_dt<DT_F32>(W, idx, B, M, V, D, scale, out, s);
}

EmbedGradWs embed_grad_carve(void* base, int64_t B, int64_t M, int64_t V, int64_t D) {
  EmbedGradWs w{};
  char* p = (char*)base;
  size_t o = 0;
  auto take = [&](size_t bytes) {
    char* r = p ? p + o : nullptr;
    o = (o + bytes + 255) & ~size_t(255);
    return r;
  };
  const int64_t chunks = (M + RADIX_CHUNK - 1) / RADIX_CHUNK;
  for (int i = 0; i < 2; ++i) {
    w.sort.keys[i] = (int32_t*)take((size_t)(B * M) * 4);
    w.sort.vals[i] = (int32_t*)take((size_t)(B * M) * 4);
  }
  w.sort.hist = (int32_t*)take((size_t)(B * RADIX_MAX_R * chunks) * 4);
  w.sort.bins = (int32_t*)take((size_t)(B * RADIX_MAX_R) * 4);
  w.sort.total = (int32_t*)take((size_t)B * 4);
  // slices of at least SUM_MIN positions
  w.carry = (float*)take((size_t)(B * ((M + SUM_MIN - 1) / SUM_MIN) * 2 * D) * 4);
  w.total = o;
  return w;
}

hipError_t launch_embed_grad(const void* G, int gdt, const int32_t* idx, int64_t B, int64_t M,
                             int64_t V, int64_t D, float scale, bool accumulate, void* dW, int wdt,
                             const EmbedGradWs& w, hipStream_t s) {
  const int64_t bytes = accumulate ? 0 : B * V * D * dt_bytes(wdt);
  hipError_t e;
  if (B * M * M <= (int64_t)1 << 26 && M <= 8192) {  // see rank_kernel
    const int64_t nrank = (M + RANK_P - 1) / RANK_P, per = RANK_T * 16 * B;
    const int64_t nzero = (bytes + per - 1) / per;
    rank_kernel<<<dim3((unsigned)(nrank + nzero), (unsigned)B), RANK_T, 0, s>>>(
        idx, (int)M, (int)V, w.sort.keys[0], w.sort.vals[0], w.sort.total, (int)nrank, (char*)dW,
        bytes);
    e = hipGetLastError();
  } else {
    e = launch_token_sort(idx, B, M, V, w.sort, s);
    constexpr int64_t most = MAX_BLOCKS * 256;  // 16-byte pieces of a launch
    for (int64_t from = 0; e == hipSuccess && from * 16 < bytes; from += most) {
      const int64_t n = std::min<int64_t>((bytes + 15) / 16 - from, most);
      zero_kernel<<<dim3((unsigned)((n + 255) / 256)), 256, 0, s>>>((char*)dW, bytes, from);
      e = hipGetLastError();
    }
  }
  if (e != hipSuccess) return e;
  if (gdt == DT_F32)
    return launch_sums_wt<DT_F32, DT_F32>(G, B, M, V, D, scale, accumulate, dW, w, s);
  if (gdt == DT_BF16)
    return wdt == DT_F32
               ? launch_sums_wt<DT_BF16, DT_F32>(G, B, M, V, D, scale, accumulate, dW, w, s)
               : launch_sums_wt<DT_BF16, DT_BF16>(G, B, M, V, D, scale, accumulate, dW, w, s);
  return wdt == DT_F32
             ? launch_sums_wt<DT_F16, DT_F32>(G, B, M, V, D, scale, accumulate, dW, w, s)
             : launch_sums_wt<DT_F16, DT_F16>(G, B, M, V, D, scale, accumulate, dW, w, s);
}

}  // namespace fkm
